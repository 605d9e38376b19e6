// C ABI of the operators that train a map: argument checks and launches.  See
// include/bhtsne.h for the contract of each call.
#include "bhtsne.h"

#include <cmath>

#include "map.hpp"

using namespace bht;

namespace {

bool type_ok(int t) { return t == BHTSNE_F32 || t == BHTSNE_F16 || t == BHTSNE_BF16; }

bool elem_aligned(const void *p, int type)
{
    return (reinterpret_cast<uintptr_t>(p) & uintptr_t(elem_bytes(Elem(type)) - 1)) == 0;
}

constexpr int64_t kMost = (int64_t(1) << 31) - 1;

bool norm_sizes_ok(int64_t n, int64_t d) { return n >= 0 && n <= kMost && d >= 1 && d <= kNormMaxFeatures; }

// a matrix the call reads: one row may stand for all of them
bool input_ok(const void *p, int64_t stride, int64_t n, int64_t d, int type)
{
    return (p || n == 0) && elem_aligned(p, type) && (stride == 0 || (stride >= d && stride <= kMost));
}
bool output_ok(const void *p, int64_t stride, int64_t d, int type)
{
    return elem_aligned(p, type) && stride >= d && stride <= kMost;
}

bool workspace_ok(const void *ws, size_t bytes, size_t need)
{
    return ws && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0 && bytes >= need;
}

bool matrices_ok(const bhtsne_matrices *x, int64_t batch, int64_t rows, int64_t cols, int type)
{
    if (!x || (!x->data && batch > 0) || !elem_aligned(x->data, type)) return false;
    if (x->stride < cols || x->stride > kMost) return false;
    return batch <= 1 || (x->batch_stride >= 0 && x->batch_stride < (int64_t(1) << 48));
}
// Matrices that are written must not share elements: each lies behind the one before, or their rows lie behind one
// another's, all first rows, all second rows and so on.  The sizes and strides are known to be in range.
bool apart(const bhtsne_matrices *x, int64_t batch, int64_t rows, int64_t cols)
{
    if (batch <= 1 || x->batch_stride >= (rows - 1) * x->stride + cols) return true;
    return x->batch_stride >= cols && x->batch_stride <= x->stride && x->stride >= (batch - 1) * x->batch_stride + cols;
}

float power_of_two_below(double x) { return float(std::exp2(std::floor(std::log2(x)))); }

// By how much a step on A multiplies a small error of A at most: the largest derivative of t B(t)^2, which takes an
// eigenvalue t of A to the next, B(t) = a + b t + c t^2; `most` bounds t.
double growth(const double *q, double most)
{
    constexpr int kPoints = 16;
    double g = 0.0;
    for (int i = 0; i <= kPoints; ++i) {
        const double t = most * i / kPoints, b = q[0] + q[1] * t + q[2] * t * t;
        g = std::fmax(g, std::fabs(b * (b + 2.0 * t * (q[1] + 2.0 * q[2] * t))));
    }
    return g;
}

// The scales of every step.  Singular values of X start in [0, 1]; `most` bounds
// them through the steps, and with them every value of X (most), of A = X X^T
// (most^2) and of B = b A + c A^2 (b t + c t^2's largest on [0, most^2]).  Half of what fp16
// holds is kept for rounding errors' growth.  X's bound is followed down to
// 2^-110, those of A and B, which do not count beside a X when they are small, to 2^-60.
bool plan_steps(const double *coefficients, int steps, OrthSteps *plan)
{
    constexpr double kRoom = 32768.0;
    constexpr double kLeast = 0x1p-110, kLeastSquare = 0x1p-60;
    double most = 1.0, noise = 1.0, grown = 1.0;
    plan->noise = plan->reach = 1.0;
    for (int k = 0; k < steps; ++k) {
        plan->noise = std::fmax(plan->noise, noise);
        plan->reach = std::fmax(plan->reach, grown / std::fmax(most, kLeast));
        const double usual[3] = {3.4445, -4.7750, 2.0315};
        const double *q = coefficients ? coefficients + 3 * k : usual;
        if (!std::isfinite(q[0]) || !std::isfinite(q[1]) || !std::isfinite(q[2])) return false;
        const double t1 = most * most;
        const auto poly = [&](double t) { return std::fabs(q[1] * t + q[2] * t * t); };
        const auto next = [&](double t) { return std::fabs(std::sqrt(t) * (q[0] + q[1] * t + q[2] * t * t)); };
        double b = poly(t1), x = next(t1), g = std::fmax(std::fabs(q[0]), std::fabs(q[0] + q[1] * t1 + q[2] * t1 * t1));
        // extremes inside: of b t + c t^2, and of s (a + b s^2 + c s^4), both in t = s^2
        const double tb = -q[1] / (2.0 * q[2]);
        if (tb > 0.0 && tb < t1) {
            b = std::fmax(b, poly(tb));
            g = std::fmax(g, std::fabs(q[0] + q[1] * tb + q[2] * tb * tb));
        }
        const double disc = 9.0 * q[1] * q[1] - 20.0 * q[0] * q[2];
        const double roots[3] = {(-3.0 * q[1] + std::sqrt(disc)) / (10.0 * q[2]),
                                 (-3.0 * q[1] - std::sqrt(disc)) / (10.0 * q[2]), -q[0] / (3.0 * q[1])};
        for (double t : roots)
            if (t > 0.0 && t < t1) x = std::fmax(x, next(t));
        OrthStep &s = plan->step[k];
        s.a = q[0];
        s.b = q[1];
        s.c = q[2];
        s.sx = power_of_two_below(kRoom / std::fmax(most, kLeast));
        s.sa = power_of_two_below(kRoom / std::fmax(t1, kLeastSquare));
        s.sb = power_of_two_below(kRoom / std::fmax(b, kLeastSquare));
        if (!(x < 64.0)) return false;
        most = x;
        grown *= g;
        noise = growth(q, t1) * noise + most * most; // and the next A's own rounding
    }
    plan->count = steps;
    return true;
}

int orthogonal_call(OrthArgs &a, const bhtsne_matrices *G, const bhtsne_matrices *W, int64_t batch, int64_t rows,
                    int64_t cols, int type, const double *coefficients, int steps, double eps, void *workspace,
                    size_t workspace_bytes, hipStream_t stream)
{
    const size_t need = bhtsne_orthogonalise_workspace_size(batch, rows, cols);
    if (need == 0 || !type_ok(type)) return BHTSNE_EINVAL;
    if (!matrices_ok(G, batch, rows, cols, type) || !matrices_ok(W, batch, rows, cols, type)) return BHTSNE_EINVAL;
    if (!apart(W, batch, rows, cols)) return BHTSNE_EINVAL;
    if (steps < 1 || steps > kOrthMaxSteps || !std::isfinite(eps) || eps < 0.0) return BHTSNE_EINVAL;
    OrthSteps plan;
    if (!plan_steps(coefficients, steps, &plan)) return BHTSNE_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return BHTSNE_EWORKSPACE;
    a.G = G->data;
    a.g_stride = G->stride;
    a.g_batch = G->batch_stride;
    a.W = W->data;
    a.w_stride = W->stride;
    a.w_batch = W->batch_stride;
    a.batch = batch;
    a.rows = rows;
    a.cols = cols;
    a.type = Elem(type);
    a.eps = eps;
    launch_orthogonalise(a, plan, workspace, stream);
    return hipGetLastError() == hipSuccess ? BHTSNE_OK : BHTSNE_EDEVICE;
}

} // namespace

extern "C" {

int bhtsne_layer_norm(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t n, int64_t d,
                      double eps, int type, int param_type, void *y, int64_t y_stride, float *mean, float *rstd,
                      hipStream_t stream)
{
    if (!norm_sizes_ok(n, d) || !type_ok(type) || !type_ok(param_type)) return BHTSNE_EINVAL;
    if (!std::isfinite(eps) || eps < 0.0) return BHTSNE_EINVAL;
    if (!input_ok(x, x_stride, n, d, type) || (!y && n > 0) || !output_ok(y, y_stride, d, type)) return BHTSNE_EINVAL;
    if (!elem_aligned(weight, param_type) || !elem_aligned(bias, param_type)) return BHTSNE_EINVAL;
    if (!elem_aligned(mean, BHTSNE_F32) || !elem_aligned(rstd, BHTSNE_F32)) return BHTSNE_EINVAL;
    NormArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.weight = weight;
    a.bias = bias;
    a.out = y;
    a.out_stride = y_stride;
    a.mean = mean;
    a.rstd = rstd;
    a.n = n;
    a.d = d;
    a.eps = eps;
    a.type = Elem(type);
    a.param = Elem(param_type);
    launch_layer_norm(a, stream);
    return hipGetLastError() == hipSuccess ? BHTSNE_OK : BHTSNE_EDEVICE;
}

size_t bhtsne_layer_norm_workspace_size(int64_t n, int64_t d)
{
    if (!norm_sizes_ok(n, d)) return 0;
    return (size_t(norm_back_blocks(n, d)) * 2 * size_t(d) * sizeof(float) + 255) / 256 * 256;
}

int bhtsne_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                               const void *weight, const float *mean, const float *rstd, int64_t n, int64_t d,
                               int type, int param_type, void *dx, int64_t dx_stride, void *dweight, void *dbias,
                               void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!norm_sizes_ok(n, d) || !type_ok(type) || !type_ok(param_type)) return BHTSNE_EINVAL;
    if (!input_ok(dy, dy_stride, n, d, type) || !input_ok(x, x_stride, n, d, type)) return BHTSNE_EINVAL;
    if (n > 0 && (!mean || !rstd)) return BHTSNE_EINVAL;
    if (!elem_aligned(mean, BHTSNE_F32) || !elem_aligned(rstd, BHTSNE_F32)) return BHTSNE_EINVAL;
    if (!dx && !dweight && !dbias) return BHTSNE_EINVAL;
    if (dx && !output_ok(dx, dx_stride, d, type)) return BHTSNE_EINVAL;
    if (!elem_aligned(weight, param_type) || !elem_aligned(dweight, param_type) || !elem_aligned(dbias, param_type))
        return BHTSNE_EINVAL;
    const bool params = dweight || dbias;
    if (params && !workspace_ok(workspace, workspace_bytes, bhtsne_layer_norm_workspace_size(n, d)))
        return BHTSNE_EWORKSPACE;
    NormArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.dy = dy;
    a.dy_stride = dy_stride;
    a.weight = weight;
    a.out = dx;
    a.out_stride = dx_stride;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.part = params ? static_cast<float *>(workspace) : nullptr;
    a.n = n;
    a.d = d;
    a.type = Elem(type);
    a.param = Elem(param_type);
    a.dweight = dweight;
    a.dbias = dbias;
    launch_layer_norm_backward(a, stream);
    return hipGetLastError() == hipSuccess ? BHTSNE_OK : BHTSNE_EDEVICE;
}

size_t bhtsne_orthogonalise_workspace_size(int64_t batch, int64_t rows, int64_t cols)
{
    if (batch < 0 || batch > 65535 || rows < 1 || rows > kOrthMaxSide || cols < 1 || cols > kOrthMaxSide) return 0;
    return size_t(batch > 0 ? batch : 1) * orth_workspace(rows, cols);
}

int bhtsne_orthogonalise(const bhtsne_matrices *G, int64_t batch, int64_t rows, int64_t cols, int type,
                         const double *coefficients, int steps, double eps, const bhtsne_matrices *O,
                         void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    OrthArgs a = {};
    return orthogonal_call(a, G, O, batch, rows, cols, type, coefficients, steps, eps, workspace, workspace_bytes,
                           stream);
}

int bhtsne_muon_step(const bhtsne_matrices *W, const bhtsne_matrices *G, const bhtsne_matrices *M, int64_t batch,
                     int64_t rows, int64_t cols, int type, double learning_rate, double momentum, int nesterov,
                     double weight_decay, double scale, const double *coefficients, int steps, double eps,
                     void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!std::isfinite(learning_rate) || !(learning_rate > 0.0) || !(momentum >= 0.0 && momentum < 1.0))
        return BHTSNE_EINVAL;
    if (!std::isfinite(weight_decay) || weight_decay < 0.0 || !std::isfinite(scale)) return BHTSNE_EINVAL;
    if (bhtsne_orthogonalise_workspace_size(batch, rows, cols) == 0) return BHTSNE_EINVAL; // before sizes are multiplied
    if (!matrices_ok(M, batch, rows, cols, BHTSNE_F32) || !apart(M, batch, rows, cols)) return BHTSNE_EINVAL;
    OrthArgs a = {};
    a.M = static_cast<float *>(M->data);
    a.m_stride = M->stride;
    a.m_batch = M->batch_stride;
    a.momentum = float(momentum);
    a.nesterov = nesterov ? 1.0f : 0.0f;
    a.keep = float(1.0 - learning_rate * weight_decay);
    a.rate = float(learning_rate * scale);
    return orthogonal_call(a, G, W, batch, rows, cols, type, coefficients, steps, eps, workspace, workspace_bytes,
                           stream);
}

} // extern "C"
