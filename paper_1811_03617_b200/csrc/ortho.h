// The plan of an orthogonalised update (gvq.h, gvq_ortho_*): what the host builds once and the kernels read.
#pragma once
#include <cuda_fp16.h>

#include "gvq_internal.h"

namespace gvq {
namespace ortho {

constexpr int kSteps = 5;
// The quintic step  X <- a X + (b A + c A^2) X,  A = X X^T: its coefficients push every singular value of (0, 1] to about 1 in
// five steps (Jordan's choice for the Muon optimiser: slope 3.44 at zero, values end in [0.7, 1.2]).
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kEps = 1e-7f;
// Steps whose X is kept as a sum of two halves: all but the last (ortho.cu's header has the reason).
constexpr int kExactSteps = kSteps - 1;
// Short sides up to which A, and P, are sums of two halves as well (ortho.cu's header has the reason).
constexpr int kSplitSide = 128, kSplitApply = 48;
// Scale of A and of a I + b A + c A^2 in half precision: entries of both are of order 1 (at most 3.5 + 1.2 |b| + 1.44 |c| = 12),
// those off the diagonal far smaller.
constexpr float kGramScale = 256.0f;

// Tiles of the products (ortho.cu): a pair of CTAs has 256 x kPairN, a CTA alone 128 x kSoloN.
constexpr int kPairN = 256, kSoloN = 64;
// Entries of a chunk of the element-wise passes (a multiple of 1024): small plans take shorter ones, to have work for all SMs.
constexpr int kMinChunk = 1024, kMaxChunk = 8192;

// One matrix [rows][cols] of the flat gradient.  r <= c its shorter and longer side.
struct Matrix {
    int32_t rows, cols, r, c, tall, ldx, ldr;
    int32_t chunk0, n_chunks;        // its chunks in the element-wise passes
    int64_t off;                     // in the flat buffers
    uint64_t by_cols;                // floor(2^62 / cols) + 1: n / cols = (4 n * by_cols) >> 64 for n < 2^40, cols < 2^20
    // X (two buffers, in turn), X's low halves; A, P; rows ldx or ldr entries apart
    __half *x[2], *lo, *gram, *poly;
    __half *gram_lo, *poly_lo;       // what the last two lose in half precision
    int32_t split;                   // 0: nothing, 1: A is a sum of two halves, 2: P too
    float sx;                        // scale of X in half precision
    float scale;                     // of the update
};
// A tile of a product, or a part of its contraction: stages [k0, k1) of 64 steps.  parts > 1: the parts' sums meet in the
// plan's scratch from piece `slot` on (part by part), and whoever comes last adds them up.
// Stages of products of halves follow one another: hi hi, hi lo and lo hi of A^2, P_hi X and P_lo X.
struct Tile { int32_t matrix, tm, tn, k0, k1, part, parts, slot; };
struct Chunk { int32_t matrix, index; };

enum Phase { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };
// Tensor maps of a matrix: operands (boxes of 64 x 64) and results (64 columns x 32 rows)
enum Map { kX0 = 0, kX1, kGramMap, kPolyMap, kX0Out, kX1Out, kLoOut, kGramOut, kPolyOut, kGramLoMap, kPolyLoMap,
           kGramLoOut, kPolyLoOut, kMaps };

// The tiles of a phase, in runs, one for each CTA (or pair): run i is tiles [start[i], start[i + 1]).
struct Run {
    const Tile *tiles;
    const int32_t *start;
    int runs;
};

struct Device {
    const Matrix *mats;
    const CUtensorMap *maps;         // [matrices][kMaps]
    Run run[4];                      // of each phase
    int pair;                        // which tiling the tiles are of
    int split;                       // the matrices' largest
    int n_mats;
    const Chunk *chunks;
    int chunk;                       // entries of one
    int n_chunks;
    float *partial;                  // [n_chunks] sums of squares
    float *parts;                    // sums of parts of a contraction, pieces of 32 rows x 64 columns
    int32_t *tickets;                // [n_tickets] arrivals at a piece (of a tile's first part), zero between launches
    int n_tickets;
};

// momentum = beta * momentum + g (momentum may be null), u = g + beta * momentum (nesterov) or momentum, sums of squares;
// then X = u / (|u| + eps) in half precision.
struct ElementArgs {
    const float *g;
    float *momentum;
    float beta;
    int nesterov;
};
// What the last product's result is for: w <- decay w - step * scale * O, or out = O.
struct OutputArgs {
    void *ptr;
    int dtype, update;
    float decay, step;
};

cudaError_t launch_start(cudaStream_t st, const Device &dev, const ElementArgs &a);
cudaError_t launch_product(cudaStream_t st, const Device &dev, Phase phase, int step, const OutputArgs *out,
                           int32_t *error_word, int wait_kcycles, int test_drop);

// Matrices that fit an SM or a cluster of them (ortho_small.cu): the room their short side takes, 64 or 128 (0: they do not
// fit), the CTAs of a matrix and the entries of the long side that each has.
struct SmallPlan { int room, parts, span; };
constexpr size_t kSmallSmem = 226 * 1024;
SmallPlan small_plan(int n, int r, int c, int num_sms);      // n matrices, the largest of their short and of their long sides
cudaError_t launch_small(cudaStream_t st, const Matrix *mats, int n, const SmallPlan &plan, const ElementArgs &in, const OutputArgs &out,
                         int32_t *error_word, int wait_kcycles, int test_drop);

}  // namespace ortho
}  // namespace gvq
