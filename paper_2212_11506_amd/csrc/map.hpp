// Internal declarations of the operators that train a map from features to
// the embedding: layer norm over all points, and the orthogonalised momentum
// step of its weight matrices.
#pragma once

#include "common.hpp"

namespace bht {

typedef _Float16 f16;
typedef __bf16 bf16;

// element types of the C ABI (BHTSNE_F32, BHTSNE_F16, BHTSNE_BF16)
enum class Elem { kF32 = 0, kF16 = 1, kBF16 = 2 };
inline int elem_bytes(Elem e) { return e == Elem::kF32 ? 4 : 2; }

constexpr int kCus = 256; // compute units of the card

// ---------------------------------------------------------------- layer norm
// Rows of up to kNormLane kNormMaxThreads features (kNormLaneBack of them backward) are held in registers; longer rows
// are read again from the caches for each pass.
constexpr int kNormLane = 16;                      // features of a lane, forward
constexpr int kNormLaneBack = 8;                   // ... and backward
constexpr int kNormAlone = 8;                      // rounds of a block of kNormMaxThreads that make a join not worth it
constexpr int64_t kNormFewRows = 8192;             // rows that do not fill the chip at several vectors a lane
constexpr int kNormFewFeatures = 2048;             // ... and are shared out over more lanes in rows up to this
constexpr int kNormMaxThreads = 1024;              // lanes of a row
constexpr int64_t kNormStream = int64_t(256) << 20; // bytes of x from which rows do not stay in the last cache
constexpr int64_t kNormMaxFeatures = int64_t(1) << 24;
constexpr int kNormBackRows = 4;                   // backward: rows at least of a block that has one row at a time
constexpr int kNormBackThreads = 1024;             // backward: threads of a CU, whose blocks write a partial row each
// lanes of a row of d features backward, in a block of its own from 64 kNormLaneBack features on (smaller rows share
// blocks of 256)
inline int norm_back_block(int64_t d)
{
    const int64_t waves = (d + 64 * kNormLaneBack - 1) / (64 * kNormLaneBack);
    return waves <= 1 ? 256 : waves < kNormMaxThreads / 64 ? int(waves) * 64 : kNormMaxThreads;
}
inline int64_t norm_back_blocks(int64_t n, int64_t d) // the most partial sums of the weights' gradient
{
    const int64_t most = int64_t(kCus) * kNormBackThreads / norm_back_block(d);
    return n < 1 ? 1 : n < most ? n : most;
}

struct NormArgs {
    const void *x;
    const void *dy;     // backward
    const void *weight; // nullable
    const void *bias;   // nullable (forward)
    void *out;          // y, or dx (nullable in the backward pass)
    float *mean, *rstd; // written by the forward pass (nullable), read by the backward pass
    float *part;        // backward: [blocks][2][d] partial sums, nullable (no weight gradient wanted)
    void *dweight, *dbias; // backward, each nullable
    bool alone;         // backward: one block, which writes the weights' gradients itself
    int64_t x_stride, dy_stride, out_stride;
    int64_t n, d;
    double eps;
    Elem type, param;
};
void launch_layer_norm(const NormArgs &a, hipStream_t st);
// at most norm_back_blocks(n, d) partial rows are written
void launch_layer_norm_backward(const NormArgs &a, hipStream_t st);

// ------------------------------------------------------- orthogonalised update
// Newton-Schulz steps on `batch` matrices U of rows x cols.  U is kept in fp16
// planes (high and low halves) scaled by powers of two, in its own orientation
// and transposed, padded with zeros to whole tiles.
constexpr int kOrthMaxSteps = 32;
constexpr int kOrthNormBlocks = 512; // partial sums of squares of a matrix
constexpr int64_t kOrthMaxSide = 65536;

struct OrthStep {
    double a, b, c;    // X' = a X + (b A + c A A) X
    float sx, sa, sb;  // powers of two: scales of X, A and B (the polynomial) in this step
};

struct OrthArgs {
    const void *G;
    float *M;      // nullable: momentum, fp32, updated in place
    void *W;       // output: the orthogonal factor, or (M given) the weights, updated in place
    int64_t g_stride, g_batch, m_stride, m_batch, w_stride, w_batch; // in elements: between rows, between matrices
    int64_t batch, rows, cols;
    double eps;
    float momentum, nesterov, keep, rate; // W <- keep W - rate X
    Elem type;
    bool g_vec, m_vec;                    // G and M are aligned for 16-byte loads
};

struct OrthSteps {
    int count;
    double reach; // how far a small X can grow beyond the bound of its step: the largest of prod |B| / most over the steps
    double noise; // of stepping on A = X X^T alone: what a rounding error in A grows to, times itself
    OrthStep step[kOrthMaxSteps];
};

constexpr int64_t kNarrow = 64;    // directions of a narrow matrix, which is stepped in fp64 on its Gram matrix
constexpr int kNarrowSlice = 128;  // columns in LDS of one that takes two launches
constexpr int kNarrowSlices = 32;  // partial Gram matrices
inline bool orth_narrow(int64_t rows, int64_t cols) { return (rows < cols ? rows : cols) <= kNarrow; }
// ... as long as its rounding errors, 2^-53 of A at first, grow to 1e-7 of A or less; beyond, X itself is stepped on.
// Nine steps of the usual coefficients are the last (on low-rank inputs 2e-8 against 64 bits or less, less than an fp32
// rounding; ten steps would be off by 2e-7, twelve by 5e-6, sixteen by all).
constexpr double kNarrowNoise = 1e9;

struct NarrowLayout {
    int tiles;     // 16-row tiles of the shorter side
    int width;     // columns of U in LDS, a power of two
    int slices;    // partial Gram matrices (0: one block, one launch)
    size_t stride; // bytes of one matrix' workspace: the partial Gram matrices
};
NarrowLayout make_narrow_layout(int64_t rows, int64_t cols);

// Narrow matrices of many steps: X in fp64, shorter side first, without gaps, and its partial Gram matrices
constexpr int kDirect = 64;       // columns of X at a time
constexpr int kDirectSlices = 32; // partial Gram matrices
struct DirectLayout {
    int m, slices;
    int64_t n;
    size_t norm, gram, x, stride;
};
DirectLayout make_direct_layout(int64_t rows, int64_t cols);

struct OrthLayout {
    int64_t m, n;         // shorter and longer side, padded
    int64_t rows, cols;   // padded sides in the caller's orientation
    size_t u[2], v[2];    // U and its transpose, two buffers each: high plane, low plane behind it
    size_t a, b;          // A and B, planes as above
    size_t norm;          // kOrthNormBlocks doubles
    size_t lift;          // a float: 1 / the power of two that X is held larger by
    size_t stride;        // bytes of one matrix' workspace
};
OrthLayout make_orth_layout(int64_t rows, int64_t cols);
size_t orth_workspace(int64_t rows, int64_t cols); // bytes for one matrix
void launch_orthogonalise(const OrthArgs &a, const OrthSteps &steps, void *ws, hipStream_t st);

} // namespace bht
