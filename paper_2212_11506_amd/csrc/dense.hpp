// Internal declarations of the dense operators of a trained map: gated hidden
// layers, products of 8-bit integers, and the loss from neighbour lists.
#pragma once

#include "map.hpp"

namespace bht {

// ------------------------------------------------------- loss from neighbour lists
constexpr int64_t kDistilMaxList = 2048;       // listed neighbours of a row: 16 bytes of LDS each
constexpr int64_t kDistilSplit = 8192;         // values of a row at least that a block takes, of rows that are shared out
constexpr int64_t kDistilBlocks = 2048;        // blocks that fill the chip: rows are shared out below so many
constexpr int64_t kDistilWave = 2048;          // rows up to this are a wave's, longer ones a block's
// Backward: |lse| up to which the rounded lse is good enough, being off by 2^-21 at most, 8 units of the exponentials' own
// roundings, which are 16 and more.  (There the gradient is the same bits with what was kept and without.)
constexpr float kDistilNear = 16.0f;

// blocks that share a row of v logits, of n rows
inline int distil_parts(int64_t n, int64_t v)
{
    const int64_t most = (v + kDistilSplit - 1) / kDistilSplit, want = n > 0 ? kDistilBlocks / n : 1;
    return int(want < 1 ? 1 : want < most ? want : most);
}

struct DistilArgs {
    const void *logits;  // n x v
    const int32_t *idx;  // n x k
    const void *teacher; // n x k
    const float *dloss;  // backward
    const float *lse_in; // backward
    float *loss, *lse;   // forward, each nullable
    float *kept;         // forward, nullable: n x 2, a row's largest logit and its sum of exponentials
    const float *kept_in; // backward, nullable
    void *out;           // backward: n x v, may be logits
    float2 *part;        // forward: (largest logit, sum) of each part of a row
    int64_t stride, idx_stride, teacher_stride, out_stride;
    int64_t n, v;
    int32_t k, parts;
    double temperature;
    Elem type;
    bool wide_teacher; // fp32, else of `type`
};
void launch_distil_loss(const DistilArgs &a, hipStream_t st);
void launch_distil_loss_backward(const DistilArgs &a, hipStream_t st);

// ------------------------------------------------------------------- products
// Tiles that a product is made of, and the parts that its sums are shared out over
enum class Side { kSmall = 64, kMiddle = 128, kLarge = 256 };
struct Plan {
    Side side;
    int splits; // 1: none
};
constexpr int kMostSplits = 64;
constexpr int64_t kMostPart = int64_t(1) << 29; // bytes of partial sums
// rows x columns of output, of `slices` slices of K each; wide: fp32 operands.  may_split: partial sums have a place;
// most: the largest side that may be taken (256 of aligned operands).
Plan plan_product(int64_t rows, int64_t columns, int64_t slices, bool wide, bool may_split, Side most);

// Whether a product of more than a few points has so few tiles that its slices are better shared out over the waves of blocks
// of kFewRows points x 16 features: while there is a CU for each block.  Then 64 x 1024 to 512 takes 19.5 us for 27.7 (fp32),
// 8.0 for 9.1 (bf16) and 4.9 for 6.8 (8 bits), tiles' figures second; with two blocks a CU, 256 x 512 to 2048, 21.8 for 17.8,
// 9.9 for 7.0 and 6.9 for 5.8.  Rows off 16 bytes of narrow types are put together from more loads, which a tile's blocks do
// once for 64 features: 128 x 777 to 250 bf16 14.6 us for 10.7 (fp32 18.6 for 23.5).
constexpr int kFewRows = 64;
inline bool few_tiles(int64_t n, int64_t f, bool whole_pieces)
{
    return whole_pieces && (n + kFewRows - 1) / kFewRows * ((f + 15) / 16) <= 256;
}

// ---------------------------------------------------------------- gated layers
enum class Act { kSilu = 0, kGelu = 1 };

struct GatedArgs {
    const void *x, *gate, *up; // n x d, f x d
    void *h, *a, *b;           // n x f; a and b nullable
    int64_t x_stride, gate_stride, up_stride, h_stride, a_stride, b_stride;
    int64_t n, d, f;
    Act act;
    Elem type;
};
void launch_gated_layer(const GatedArgs &a, hipStream_t st);

// Backward: da and db side by side (n rows), x with padded rows, the weights transposed and side by side; partial sums of
// the weights' gradients where they are shared out over the points.
constexpr int64_t pad16(int64_t count, int bytes) { return (count * bytes + 15) / 16 * 16 / bytes; }
struct GatedBackLayout {
    int64_t fp, dp;  // padded f and d: to whole slices, and to 16 bytes
    int64_t np;      // points, padded to whole slices
    int64_t ld;      // values from row to row of da and db
    Plan x, weights; // of dx, and of the weights' gradients
    bool wide;       // operands in fp32
    size_t d, xp, wt, part, total;
};
GatedBackLayout make_gated_back_layout(int64_t n, int64_t d, int64_t f, Elem type);

struct GatedBackArgs {
    const void *dh, *x, *gate, *up, *a, *b;
    void *dx, *dgate, *dup; // each nullable
    int64_t dh_stride, x_stride, gate_stride, up_stride, a_stride, b_stride, dx_stride, dgate_stride, dup_stride;
    int64_t n, d, f;
    Act act;
    Elem type;
    void *ws;
};
void launch_gated_layer_backward(const GatedBackArgs &a, hipStream_t st);

// ---------------------------------------------------------- products of 8-bit integers
constexpr int64_t kLinearSlice = 128;       // values of a slice of a row
constexpr int64_t kLinearMaxDepth = 131071; // (-128)^2 so many times stays below 2^31
constexpr int64_t kLinearMaxFeatures = int64_t(1) << 26; // a launch has fewer than 2^32 threads: 512 for 16 features

// A few points, which their product quantises itself (kFewValues values, with the rows' padding)
constexpr int64_t kFewPoints = 16, kFewValues = 8192;
inline bool linear_few(int64_t n, int64_t d)
{
    return n <= kFewPoints && n * ((d + kLinearSlice - 1) / kLinearSlice * kLinearSlice) <= kFewValues;
}

struct QuantiseArgs {
    const void *x;
    int8_t *q;
    float *scale;
    int64_t x_stride, q_stride;
    int64_t n, d;
    int64_t pad; // zeros behind each row's values, up to so many (<= q_stride)
    Elem type;
};
void launch_quantise_rows(const QuantiseArgs &a, hipStream_t st);

struct LinearArgs {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    const void *bias; // nullable
    void *out;
    int64_t x_stride, w_stride, out_stride;
    int64_t n, d, f;
    Elem type, bias_type;
    bool padded; // x's rows go on with zeros to whole slices
};
void launch_linear_i8(const LinearArgs &a, hipStream_t st);
void launch_linear_values(LinearArgs a, const QuantiseArgs &q, hipStream_t st); // of the rows that q quantises

} // namespace bht
