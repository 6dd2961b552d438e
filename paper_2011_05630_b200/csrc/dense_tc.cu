// Dense products on tcgen05 by CTA pairs: one persistent kernel for the forward products (with their epilogues) and the gradients'.
//
// A pair works on a 256 x BN tile of the result: either CTA loads its own 128 rows of A and half of B's rows, the tensor cores
// of both read both halves of B (cta_group::2), so that an SM's shared memory takes in 32 KB per 64 of K for 2 * 128 * 256 * 64
// operations (BN = 256) - half of what a CTA of its own would need.  One accumulator of BN columns of tensor memory is filled while the other
// is drained.  A gated tile is the same product with the gate's 128 rows as one half of B and the up projection's as the other:
// G and U of an output lie in the same lane, BN / 2 columns apart.
//
// Operands come as they lie in memory, along K or across it (the backward products read weights, inputs and gradients as the
// forward pass left them; nothing is transposed): an operand across K arrives as boxes of 64 values of its other index by 64 of K.
#include <cuda.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_tc.cuh"

namespace dlf {

namespace {

constexpr int kEpiWarps = 8;                // warps 0..7: warp & 3 = TMEM lane quarter, warp >> 2 = half of the columns
constexpr int kAWarp = kEpiWarps, kBWarp = kAWarp + 1, kMmaWarp = kBWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kRing = 192 * 1024;           // 6 stages of 32 KB, 8 of 24 KB
constexpr int kStaging = kEpiWarps * 4096;  // 32 rows of 64 values for each epilogue warp
constexpr int kDynSmem = kRing + kStaging + 1024;
constexpr int kMaxStages = 8;
enum { EPI_PLAIN = 0, EPI_LINEAR = 1, EPI_GATED = 2 };

// One product, or the two gradients' products that share a launch (JOBS = 2): the input's first, whose K is the longer one or not.
struct PairJob {
    CUtensorMap a[2], b[2], out[3];
    Mat o[3];                     // (rows off the 16-byte boundaries have no tensor map)
    long long M, N, tiles, group_tiles;
    int tiles_m, tiles_n;
    int chunks1, chunks;          // 64-value chunks of K: of the first source, of both
    int groups;
    bool amn, out_tma[3];
};
template <int JOBS>
struct PairParams {
    PairJob job[JOBS];
    Mat res;
    const float* bias[2];
    int act;
    bool res_vec;
    // Pairs take the first job's tiles in turn; `rest` of them have one more of these than the others, and with it `many` of the second job's
    // tiles where the others have `few` (the host weighs the tiles).
    int pairs, rest, few, many;
};

// The i-th tile of a pair; false behind its last one.
template <int JOBS>
__device__ __forceinline__ bool tile_of(const PairParams<JOBS>& p, int pair, int i, int* job, long long* t) {
    *job = 0;
    *t = pair + static_cast<long long>(i) * p.pairs;
    if (*t < p.job[0].tiles) return true;
    if (JOBS == 1) return false;
    *job = JOBS - 1;
    const bool first = pair < p.rest;
    i -= static_cast<int>(p.job[0].tiles / p.pairs) + (first ? 1 : 0);
    const int others = p.pairs - p.rest;
    *t = first ? static_cast<long long>(p.few) * others + static_cast<long long>(i) * p.rest + pair : static_cast<long long>(i) * others + pair - p.rest;
    return i < (first ? p.many : p.few) && *t < p.job[JOBS - 1].tiles;
}

// Tiles are numbered along n within bands of kBand rows of tiles, so that the pairs at work at one time share operands.
constexpr int kBand = 8;
struct TileAt { int group; long long m0, n0; };
template <int BN, int EPI>
__device__ __forceinline__ TileAt tile_at(const PairJob& p, long long t) {
    TileAt r;
    r.group = p.groups > 1 && t >= p.group_tiles ? 1 : 0;
    t -= r.group ? p.group_tiles : 0;
    const long long per_band = static_cast<long long>(kBand) * p.tiles_n, band = t / per_band, in = t - band * per_band;
    const int rows = min(kBand, p.tiles_m - static_cast<int>(band) * kBand);
    const long long n = in / rows;
    r.m0 = (band * kBand + (in - n * rows)) * 256;
    r.n0 = n * (EPI == EPI_GATED ? BN / 2 : BN);
    return r;
}

// ---- a warp's rows between registers and memory ----
// Rows that start anywhere into a warp's staging buffer, a row's columns side by side; zeros behind `rows` and `cols`.
__device__ __noinline__ void rows64_in(const unsigned short* p, int64_t ld, uint8_t* stg, int lane, int rows, int cols) {
#pragma unroll 8
    for (int r = 0; r < 32; r++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int c = lane + h * 32;
            const unsigned short v = r < rows && c < cols ? ld_map(p + r * ld + c) : static_cast<unsigned short>(0);
            *reinterpret_cast<unsigned short*>(stg + r * 128 + (((c >> 3) ^ (r & 7)) << 4) + (c & 7) * 2) = v;
        }
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
    rows64_in(p, m.ld, stg, lane, rows, cols);
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

// A warp's staged rows (`rows` of 32, the first `cols` of 64 values) to rows that start anywhere, in memory's pieces of 16 bytes: of a row's 64
// values the first ones up to a piece's start and the last ones, eight together, leave one by one, seven pieces between them
// whole.  (Out of line: its registers are not the other path's.)
__device__ __noinline__ void rows64_out(unsigned short* p0, int64_t ld, const uint8_t* stg, int lane, int rows, int cols) {
    const auto head = [](const unsigned short* p) { return static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) >> 1)) & 7u); };
    const auto at = [&](int r, int c) { return *reinterpret_cast<const unsigned short*>(stg + r * 128 + (((c >> 3) ^ (r & 7)) << 4) + (c & 7) * 2); };
#pragma unroll
    for (int it = 0; it < 7; it++) {
        const int i = it * 32 + lane, r = i / 7;
        unsigned short* const p = p0 + r * ld;
        const int c = head(p) + (i - r * 7) * 8, k = c >> 3;
        if (r >= rows || c >= cols) continue;
        if (c + 8 <= cols) {
            const uint8_t* const row = stg + r * 128;
            const uint4 a = *reinterpret_cast<const uint4*>(row + ((k ^ (r & 7)) << 4)), b = *reinterpret_cast<const uint4*>(row + (((k + 1) & 7) ^ (r & 7)) * 16);
            *reinterpret_cast<uint4*>(p + c) = shift16(a, b, static_cast<uint32_t>(c & 7) * 2);
        } else {
            for (int e = c; e < cols; e++) p[e] = at(r, e);
        }
    }
#pragma unroll
    for (int it = 0; it < 8; it++) {
        const int i = it * 32 + lane, r = i >> 3, e = i & 7;
        unsigned short* const p = p0 + r * ld;
        const int c = e < head(p) ? e : 56 + e;
        if (r < rows && c < cols) p[c] = at(r, c);
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
        rows64_out(static_cast<unsigned short*>(const_cast<void*>(o.p)) + row0 * o.ld + col0, o.ld, stg, lane, static_cast<int>(min(static_cast<int64_t>(32), rows_end - row0)), cols);
        __syncwarp();
    }
}

template <typename T, int EPI, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) dense_pair_kernel(const __grid_constant__ PairParams<EPI == EPI_PLAIN ? 2 : 1> p) {
    constexpr bool BMN = EPI == EPI_PLAIN;   // (a forward product's operands lie along K; of the gradients' B lies across, and A, too, for weights)
    constexpr int kABytes = 128 * 128, kBRows = BN / 2, kBBytes = kBRows * 128, kStageBytes = kABytes + kBBytes, kStages = kRing / kStageBytes;
    static_assert(kStages <= kMaxStages, "ring");
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sbase = smem_raw + (base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_rank());
    volatile int* abort_flag = &abort_s;
    int* status = g_dense_status;
    const int pair = static_cast<int>(blockIdx.x) >> 1;
    int ji = 0;          // a tile's job and number
    long long t = 0;

    if (warp == 0) {
        if (lane == 0) abort_s = 0;
        if (lane < kStages) {
            mbar_init(&full_bar[lane], 2);    // the A and the B producer of the pair's first CTA, each with both CTAs' bytes
            mbar_init(&empty_bar[lane], 1);
        }
        if (lane < 2) {
            mbar_init(&tfull_bar[lane], 1);
            mbar_init(&tempty_bar[lane], 2 * kEpiWarps);
        }
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc_pair(&tmem_base_s, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive();   // both CTAs' barriers are initialised before either is signalled
    cluster_wait();
    tc_fence_after_sync();
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t tmem_base = tmem_base_s;

    if (warp == kAWarp || warp == kBWarp) {
        // ---- producers: one warp for A, one for B; the copies of a stage complete on the first CTA's barrier ----
        const bool is_b = warp == kBWarp;
        const uint32_t my_bytes = is_b ? kBBytes : kABytes;
        int st = 0;
        uint32_t ph = 0;
        bool ok = true;
#pragma unroll 1
        for (int i = 0; ok && tile_of(p, pair, i, &ji, &t); i++) {
            const PairJob& job = p.job[ji];
            const TileAt at = tile_at<BN, EPI>(job, t);
            const bool across = is_b ? BMN : EPI == EPI_PLAIN && job.amn;
            const int boxes = across ? (is_b ? kBRows / 64 : 2) : 1, chunks = job.chunks, chunks1 = job.chunks1;
            const int row0 = is_b ? static_cast<int>(at.n0) + (EPI == EPI_GATED ? 0 : rank * kBRows) : static_cast<int>(at.m0) + rank * 128;
            const CUtensorMap* const map0 = is_b ? &job.b[EPI == EPI_GATED ? rank : 0] : &job.a[at.group];
            const CUtensorMap* const map1 = is_b ? &job.b[1] : &job.a[1];
#pragma unroll 1
            for (int c = 0; c < chunks; c++) {
                ok = mbar_wait_warp(&empty_bar[st], ph ^ 1u, abort_flag, status, 0x100 | (blockIdx.x << 12));
                if (!ok) break;
                if (lane == 0 && rank == 0) mbar_expect_tx(&full_bar[st], 2 * my_bytes);
                __syncwarp();
                const int bx = lane - boxes * st;   // (another lane for every stage: the copies of one thread run one after the other)
                if (bx >= 0 && bx < boxes) {
                    const bool second = c >= chunks1;
                    const int k0 = (second ? c - chunks1 : c) * 64, row = row0 + bx * 64;
                    tma_load_2d_pair(sbase + st * kStageBytes + (is_b ? kABytes : 0) + bx * 8192, second ? map1 : map0, mapa(smem_u32(&full_bar[st]), 0),
                                     across ? row : k0, across ? k0 : row);
                }
                __syncwarp();
                if (++st == kStages) { st = 0; ph ^= 1u; }
            }
        }
    } else if (warp == kMmaWarp) {
        // ---- issuer: the pair's first CTA, the whole warp walks the loop, one elected lane issues ----
        if (rank == 0) {
            const uint32_t b0 = BMN ? umma_desc_mn_lo(base + kABytes, 8192) : umma_desc_lo(base + kABytes);
            int st = 0;
            uint32_t ph = 0, j = 0;
            bool ok = true;
#pragma unroll 1
            for (; ok && tile_of(p, pair, static_cast<int>(j), &ji, &t); j++) {
                const PairJob& job = p.job[ji];
                const bool amn = EPI == EPI_PLAIN && job.amn;
                const int chunks = job.chunks;
                const uint32_t acc = j & 1u;
                ok = mbar_wait_warp(&tempty_bar[acc], ((j >> 1) & 1u) ^ 1u, abort_flag, status, 0x200 | (blockIdx.x << 12));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + acc * 256u;
                auto multiply = [&](auto across) {   // (a loop for each kind of operand A: a step that is no constant costs 5 % of the weights' gradients)
                    constexpr bool AMN = across.value;
                    constexpr uint32_t idesc = dense_idesc<T>(256, BN, AMN, BMN);
                    const uint32_t a0 = AMN ? umma_desc_mn_lo(base, 8192) : umma_desc_lo(base);
#pragma unroll 1
                    for (int c = 0; c < chunks; c++) {
                        ok = mbar_wait_warp<true>(&full_bar[st], ph, abort_flag, status, 0x300 | (blockIdx.x << 12));
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint32_t off = static_cast<uint32_t>(st) * (kStageBytes >> 4);
                        if (elect_one()) {
                            umma_chunk<2, AMN, BMN>(d_tmem, a0 + off, b0 + off, idesc, c != 0);
                            umma_commit_pair(&empty_bar[st]);
                        }
                        __syncwarp();
                        if (++st == kStages) { st = 0; ph ^= 1u; }
                    }
                };
                if (amn) multiply(std::integral_constant<bool, EPI == EPI_PLAIN>{});
                else multiply(std::false_type{});
                if (ok && elect_one()) umma_commit_pair(&tfull_bar[acc]);
                __syncwarp();
            }
        }
    } else {
        // ---- epilogue: a lane holds a row of the tile; 64 columns at a time go through the warp's staging buffer (rows of 128
        // bytes, swizzled as the tensor map expects, which also keeps the lanes' 16-byte writes apart) and leave as one TMA store ----
        const int q = warp & 3, half = warp >> 2;
        uint8_t* stg = sbase + kRing + warp * 4096;
        constexpr int kChunks = EPI == EPI_GATED ? BN / 256 : BN / 128;   // of 64 output columns, for each warp
        static_assert(kChunks >= 1, "tile");
        uint32_t j = 0;
        bool ok = true;
#pragma unroll 1
        for (; ok && tile_of(p, pair, static_cast<int>(j), &ji, &t); j++) {
            const PairJob& job = p.job[ji];
            const TileAt at = tile_at<BN, EPI>(job, t);
            const uint32_t acc = j & 1u;
            const long long row0 = at.m0 + rank * 128 + q * 32;
            const uint32_t taddr = tmem_base + acc * 256u + (static_cast<uint32_t>(q * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < kChunks; c++) {
                const int cc = half * (kChunks * 64) + c * 64;      // column within the tile's outputs
                const long long col0 = at.n0 + cc;
                const int cols = static_cast<int>(max(0ll, min(64ll, job.N - col0)));
                uint4 res[EPI == EPI_LINEAR ? 8 : 1];
                if constexpr (EPI == EPI_LINEAR) {
                    if (p.res.p) load_rows64<T>(p.res, p.res_vec, stg, lane, row0, col0, job.M, cols, res);
                }
                if (c == 0) {
                    ok = mbar_wait_warp(&tfull_bar[acc], (j >> 1) & 1u, abort_flag, status, 0x400 | (blockIdx.x << 12));
                    tc_fence_after_sync();
                }
                if (!ok) break;
                float v[64];
                tmem_ld32(taddr + cc, v);
                tmem_ld32(taddr + cc + 32, v + 32);
                [[maybe_unused]] float u[EPI == EPI_GATED ? 64 : 1];
                if constexpr (EPI == EPI_GATED) {
                    tmem_ld32(taddr + BN / 2 + cc, u);
                    tmem_ld32(taddr + BN / 2 + cc + 32, u + 32);
                }
                if (c == kChunks - 1) {   // the accumulator has been read
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(mapa(smem_u32(&tempty_bar[acc]), 0));
                }
                if (cols == 0 || row0 >= job.M) continue;   // (the same for the whole warp)
                auto put = [&](int which, const float* val) {
                    store_rows64<T>(job.o[which], &job.out[which], job.out_tma[which], stg, lane, row0, col0, job.M, cols, val);
                };
                if constexpr (EPI == EPI_PLAIN) {
                    put(at.group, v);
                } else if constexpr (EPI == EPI_LINEAR) {
                    if (p.bias[0]) add_bias64(p.bias[0], col0, cols, v);
                    if (p.res.p) add_row64<T>(res, v);
                    if (job.o[1].p) put(1, v);
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int i = 0; i < 64; i += 2) {
                            const float2 a = act2<act.value>(make_float2(v[i], v[i + 1]));
                            v[i] = a.x; v[i + 1] = a.y;
                        }
                    });
                    put(0, v);
                } else {
                    if (p.bias[0]) add_bias64(p.bias[0], col0, cols, v);
                    if (p.bias[1]) add_bias64(p.bias[1], col0, cols, u);
                    if (job.o[1].p) put(1, v);
                    if (job.o[2].p) put(2, u);
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int i = 0; i < 64; i += 2) {
                            const float2 a = mul2(act2<act.value>(make_float2(v[i], v[i + 1])), make_float2(u[i], u[i + 1]));
                            v[i] = a.x; v[i + 1] = a.y;
                        }
                    });
                    put(0, v);
                }
            }
        }
        if (lane == 0) tma_store_wait_read();   // shared memory outlives every store that reads it
        __syncwarp();
    }
    tc_fence_before_sync();
    __syncthreads();
    // neither CTA leaves while the other may still read its operands or signal its barriers
    cluster_arrive();
    cluster_wait();
    if (warp == kMmaWarp) {
        if (abort_s) {
            if (lane == 0) dense_count_abort();
            __nanosleep(20000);
        }
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

int fill_job(const DenseGemm& g, int bn, PairJob* p) {
    int rc = DLF_OK;
    for (int i = 0; i < 2 && rc == DLF_OK; i++) {
        const Mat &a = g.a[i], &b = g.b[i];
        if (a.p) rc = g.a_mn ? dense_map(&p->a[i], a, g.K, g.M, 64, 64) : dense_map(&p->a[i], a, g.M, g.K, 128, 64);
        if (b.p && rc == DLF_OK) rc = g.b_mn ? dense_map(&p->b[i], b, g.K, g.N, 64, 64) : dense_map(&p->b[i], b, g.N, g.K, bn / 2, 64);
    }
    for (int i = 0; i < 3 && rc == DLF_OK; i++) {
        p->o[i] = g.out[i];
        p->out_tma[i] = g.out[i].p && dense_rows16(g.out[i]);
        if (p->out_tma[i]) rc = dense_map(&p->out[i], g.out[i], g.M, g.N, 32, 64);
    }
    const int step = g.gated ? bn / 2 : bn;
    p->M = g.M; p->N = g.N;
    p->tiles_m = static_cast<int>((g.M + 255) / 256);
    p->tiles_n = static_cast<int>((g.N + step - 1) / step);
    p->group_tiles = static_cast<long long>(p->tiles_m) * p->tiles_n;
    p->tiles = p->group_tiles * g.groups;
    p->chunks1 = static_cast<int>((g.K + 63) / 64);
    p->chunks = p->chunks1 * g.sources;
    p->groups = g.groups;
    p->amn = g.a_mn;
    return rc;
}
template <typename FN, typename PARAMS>
int launch_pairs(FN fn, const PARAMS& p, cudaStream_t s) {
    const int rc = dense_smem_attr(reinterpret_cast<const void*>(fn), kDynSmem);
    if (rc) return rc;
    const cudaError_t e = launch_kernel(fn, 2 * p.pairs, kThreads, kDynSmem, s, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}
template <typename T>
int launch_forward(const DenseGemm& g, int bn, const PairParams<1>& p, cudaStream_t s) {
    if (g.gated) return launch_pairs(dense_pair_kernel<T, EPI_GATED, 256>, p, s);
    return bn == 256 ? launch_pairs(dense_pair_kernel<T, EPI_LINEAR, 256>, p, s) : launch_pairs(dense_pair_kernel<T, EPI_LINEAR, 128>, p, s);
}
template <typename T>
int launch_grads(int bn, const PairParams<2>& p, cudaStream_t s) {
    return bn == 256 ? launch_pairs(dense_pair_kernel<T, EPI_PLAIN, 256>, p, s) : launch_pairs(dense_pair_kernel<T, EPI_PLAIN, 128>, p, s);
}

}  // namespace

// How the pairs share two jobs' tiles (see PairParams): the least time, in chunks of K, by which every tile has a pair.  Tiles of the second
// job go to the pairs with one tile less of the first until they are as late as the others.
DensePairShare dense_pair_share(const DenseGemm* g, int n, int bn, int sms) {
    // (a tile's rows take as long as 8 chunks, 2.4 of them before its accumulator is free again)
    auto tiles = [&](const DenseGemm& q) { return ((q.M + 255) / 256) * ((q.N + (q.gated ? bn / 2 : bn) - 1) / (q.gated ? bn / 2 : bn)) * q.groups; };
    auto cost = [&](const DenseGemm& q) { return static_cast<double>((q.K + 63) / 64 * q.sources) + 2.4; };
    const int64_t t0 = tiles(g[0]), t1 = n > 1 ? tiles(g[1]) : 0;
    const int pairs = static_cast<int>(std::min<int64_t>(t0 + t1, std::max(1, sms / 2)));
    const int64_t q0 = t0 / pairs, r = t0 % pairs;
    DensePairShare share{-1.0, pairs, static_cast<int>(r), 0, 0};
    const double c0 = cost(g[0]), end = c0 * static_cast<double>(q0 + (r ? 1 : 0));
    if (t1 == 0) {
        share.chunks = end;
        return share;
    }
    const double c1 = cost(g[1]);
    // the earliest end at which the places suffice, from the perfectly even one on
    double T = (c0 * static_cast<double>(t0) + c1 * static_cast<double>(t1)) / pairs;
    for (int i = 0; i < 1000000; i++) {
        const int64_t few_n = std::max<int64_t>(0, static_cast<int64_t>((T - c0 * static_cast<double>(q0)) / c1 + 1e-9));
        const int64_t many_n = std::max<int64_t>(0, static_cast<int64_t>((T - c0 * static_cast<double>(q0 + 1)) / c1 + 1e-9));
        if (few_n * (pairs - r) + many_n * r >= t1) {
            share.few = static_cast<int>(few_n);
            share.many = static_cast<int>(many_n);
            share.chunks = std::max(end, T);
            return share;
        }
        T += c1 / 8;
    }
    return share;
}

int launch_dense_pair(const DenseGemm* g, int n, int bn, int sms, cudaStream_t s) {
    int rc = DLF_OK;
    const DensePairShare share = dense_pair_share(g, n, bn, sms);
    if (share.chunks < 0) return DLF_E_UNSUPPORTED;
    const bool bf = g[0].dtype == DLF_BF16;
    if (!g[0].b_mn) {
        PairParams<1> p;
        std::memset(&p, 0, sizeof(p));
        rc = fill_job(g[0], bn, &p.job[0]);
        if (rc) return rc;
        p.res = g[0].res;
        p.res_vec = dense_rows16(g[0].res);
        p.bias[0] = g[0].bias[0]; p.bias[1] = g[0].bias[1];
        p.act = g[0].act;
        p.pairs = share.pairs;
        return bf ? launch_forward<__nv_bfloat16>(g[0], bn, p, s) : launch_forward<__half>(g[0], bn, p, s);
    }
    PairParams<2> p;
    std::memset(&p, 0, sizeof(p));
    for (int i = 0; i < n; i++) {
        rc = fill_job(g[i], bn, &p.job[i]);
        if (rc) return rc;
    }
    p.pairs = share.pairs;
    p.rest = share.rest; p.few = share.few; p.many = share.many;
    return bf ? launch_grads<__nv_bfloat16>(bn, p, s) : launch_grads<__half>(bn, p, s);
}

int dense_pair_gave_up(cudaStream_t s, int* count) { return dense_gave_up(s, count); }
int dense_pair_stall(unsigned long long limit_ns, cudaStream_t s) { return dense_stall(limit_ns, s); }

}  // namespace dlf
