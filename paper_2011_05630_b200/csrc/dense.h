// Dense operators (dlf_linear*, dlf_gated*): what their host side hands to the kernels.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace dlf {

// A row-major matrix of 16-bit values; ld = elements between the starts of two rows.
struct Mat {
    const void* p;
    int64_t ld;
};

// D(m, n) = sum over k of A(m, k) B(n, k), summed in fp32 and finished by an epilogue.
//   two sources:  D = A0 B0^T + A1 B1^T in one sum (the gradient of an input that two projections read)
//   two groups:   D0 = A0 B0^T and D1 = A1 B0^T as one launch (the gradients of two weight matrices that read one input)
//   gated:        G = A0 B0^T + bias0, U = A0 B1^T + bias1, out[0] = act(G) U, and G and U themselves to out[1] and out[2]
//   otherwise:    out[0] = act(D + bias0 + res), and the sum itself to out[1]
// a_mn, b_mn: the operand is stored the other way round, one row for each k.
struct DenseGemm {
    int dtype, act;
    int64_t M, N, K;
    int sources, groups;
    bool gated, a_mn, b_mn;
    Mat a[2], b[2];
    const float* bias[2];
    Mat res;
    Mat out[3];
};

// Gradients behind an activation, element by element, and their sums over the rows in fp32 (of the values before rounding):
//   gated:      d0 = dy u act'(z), d1 = dy act(z)        otherwise: d0 = dy act'(z)
// d0c: d0 once more at another place.  Any output may be null.
struct DenseGrad {
    int dtype, act;
    int64_t M, N;
    bool gated;
    Mat dy, z, u;
    Mat d0, d1, d0c;
    float *db0, *db1;
};

// True if a matrix can be a TMA operand: rows start on 16-byte boundaries.
inline bool dense_rows16(const Mat& m) { return aligned(16, m.p) && m.ld % 8 == 0; }

// Products `g[0]` to `g[n - 1]` as one launch: one forward product, or one or two gradients (b_mn).
// dense_tc.cu: tiles of 256 rows by bn (256, 128; gated: 256, both halves) columns of B; operands with rows on 16-byte boundaries.
int launch_dense_pair(const DenseGemm* g, int n, int bn, int sms, cudaStream_t s);
struct DensePairShare {
    double chunks;                // of K until the last pair is done; negative: no such share
    int pairs, rest, few, many;   // (dense_tc.cu's PairParams)
};
DensePairShare dense_pair_share(const DenseGemm* g, int n, int bn, int sms);
int dense_pair_gave_up(cudaStream_t s, int* count);           // waits for the stream; CTAs in which a bounded wait has given up so far
int dense_pair_stall(unsigned long long limit_ns, cudaStream_t s);   // a wait that does
// dense_lat.cu: tiles of at most 128 rows by `bn` columns of B (64, 128, forward 96, too; both halves of a gated tile), K shared out over `split` CTAs (1, 2,
// 4, 8).
struct DenseLatChoice {
    int bn, split;
    bool deep;   // a tile of one CTA: the whole of an SM's shared memory for its ring instead of half
};
bool dense_lat_possible(const DenseGemm& g, const DenseLatChoice& c, int* rows, int* stages, bool* two);   // `two` of its CTAs fit an SM
int launch_dense_lat(const DenseGemm* g, int n, const DenseLatChoice& c, cudaStream_t s);
int dense_lat_gave_up(cudaStream_t s, int* count);
int dense_lat_stall(unsigned long long limit_ns, cudaStream_t s);

bool dense_gemv_takes(const DenseGemm& g);                           // dense_gemv.cu: forward products of a few tokens, any rows
struct DenseGemvLayout {
    bool any;               // rows anywhere
    int rows, lg_ranks;     // weight rows of a CTA; CTAs that share their K
    int64_t groups, blocks; // CTAs without such a share; blocks of K of a CTA before it
};
DenseGemvLayout dense_gemv_layout(const DenseGemm& g, int sms);
int launch_dense_gemv(const DenseGemm& g, int sms, cudaStream_t s);

// Copies matrices to rows on 16-byte boundaries (zeros behind a row's end, up to the boundary).
constexpr int kMaxPacks = 3;   // (x and both weight matrices)
struct DensePack {
    int64_t rows, cols;
    Mat from, to;
};
int launch_dense_pack(const DensePack* jobs, int n, int sms, cudaStream_t s);
int launch_dense_grad(const DenseGrad& g, int sms, cudaStream_t s);

}  // namespace dlf
