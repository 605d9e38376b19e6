// C ABI of the dense operators of a trained map: argument checks and launches.
// See include/bhtsne.h for the contract of each call.
#include "bhtsne.h"

#include <cmath>

#include "dense.hpp"

using namespace bht;

namespace {

constexpr int64_t kMost = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxSide = 65536;

bool type_ok(int t) { return t == BHTSNE_F32 || t == BHTSNE_F16 || t == BHTSNE_BF16; }

bool aligned(const void *p, int type)
{
    const uintptr_t bytes = type == BHTSNE_I8 ? 1 : uintptr_t(elem_bytes(Elem(type)));
    return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

// a matrix the call reads: one row may stand for all of them
bool input_ok(const void *p, int64_t stride, int64_t n, int64_t d, int type)
{
    return (p || n == 0 || d == 0) && aligned(p, type) && (stride == 0 || (stride >= d && stride <= kMost));
}
bool output_ok(const void *p, int64_t stride, int64_t n, int64_t d, int type)
{
    return (p || n == 0) && aligned(p, type) && stride >= d && stride <= kMost;
}
bool workspace_ok(const void *ws, size_t bytes, size_t need)
{
    return ws && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0 && bytes >= need;
}
bool layer_sizes_ok(int64_t n, int64_t d, int64_t f)
{
    return n >= 0 && n <= kMost && d >= 1 && d <= kMaxSide && f >= 1 && f <= kMaxSide;
}
// no output is an input or another output (rows of one buffer may lie between another's, so ranges say nothing)
template <size_t kOuts, size_t kIns> bool apart(const void *const (&outs)[kOuts], const void *const (&ins)[kIns])
{
    for (size_t i = 0; i < kOuts; ++i) {
        if (!outs[i]) continue;
        for (const void *p : ins)
            if (outs[i] == p) return false;
        for (size_t k = i + 1; k < kOuts; ++k)
            if (outs[i] == outs[k]) return false;
    }
    return true;
}
bool act_ok(int act) { return act == BHTSNE_SILU || act == BHTSNE_GELU; }

int status() { return hipGetLastError() == hipSuccess ? BHTSNE_OK : BHTSNE_EDEVICE; }

bool distil_sizes_ok(int64_t n, int64_t v, int64_t k)
{
    return n >= 0 && n <= kMost && v >= 1 && v <= kMost && k >= 0 && k <= kDistilMaxList;
}

// what both directions take of a loss from neighbour lists
bool distil_inputs(DistilArgs *a, const void *logits, int64_t stride, int64_t n, int64_t v, const int32_t *idx, int64_t idx_stride,
                   const void *teacher, int64_t teacher_stride, int64_t k, double temperature, int type, int teacher_type)
{
    if (!distil_sizes_ok(n, v, k) || !type_ok(type) || (teacher_type != type && teacher_type != BHTSNE_F32)) return false;
    if (!std::isfinite(temperature) || !(temperature >= 1e-6 && temperature <= 1e6)) return false;
    if (!input_ok(logits, stride, n, v, type) || !input_ok(idx, idx_stride, n, k, BHTSNE_F32)
        || !input_ok(teacher, teacher_stride, n, k, teacher_type))
        return false;
    a->logits = logits;
    a->stride = stride;
    a->idx = idx;
    a->idx_stride = idx_stride;
    a->teacher = teacher;
    a->teacher_stride = teacher_stride;
    a->n = n;
    a->v = v;
    a->k = int32_t(k);
    a->parts = distil_parts(n, v);
    a->temperature = temperature;
    a->type = Elem(type);
    a->wide_teacher = teacher_type == BHTSNE_F32;
    return true;
}

} // namespace

extern "C" {

int bhtsne_gated_layer(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, const void *up, int64_t up_stride,
                       int64_t n, int64_t d, int64_t f, int activation, int type, void *h, int64_t h_stride, void *a,
                       int64_t a_stride, void *b, int64_t b_stride, hipStream_t stream)
{
    if (!layer_sizes_ok(n, d, f) || !act_ok(activation) || !type_ok(type)) return BHTSNE_EINVAL;
    if (!input_ok(x, x_stride, n, d, type) || !output_ok(const_cast<void *>(gate), gate_stride, f, d, type)
        || !output_ok(const_cast<void *>(up), up_stride, f, d, type))
        return BHTSNE_EINVAL;
    if (!output_ok(h, h_stride, n, f, type) || (a && !output_ok(a, a_stride, n, f, type)) || (b && !output_ok(b, b_stride, n, f, type)))
        return BHTSNE_EINVAL;
    if (n > 0 && !apart({h, a, b}, {x, gate, up})) return BHTSNE_EINVAL;
    GatedArgs g = {};
    g.x = x;
    g.x_stride = x_stride;
    g.gate = gate;
    g.gate_stride = gate_stride;
    g.up = up;
    g.up_stride = up_stride;
    g.n = n;
    g.d = d;
    g.f = f;
    g.act = Act(activation);
    g.type = Elem(type);
    g.h = h;
    g.h_stride = h_stride;
    g.a = a;
    g.a_stride = a_stride;
    g.b = b;
    g.b_stride = b_stride;
    launch_gated_layer(g, stream);
    return status();
}

size_t bhtsne_gated_layer_workspace_size(int64_t n, int64_t d, int64_t f, int type)
{
    if (!layer_sizes_ok(n, d, f) || !type_ok(type)) return 0;
    return make_gated_back_layout(n, d, f, Elem(type)).total;
}

int bhtsne_gated_layer_backward(const void *dh, int64_t dh_stride, const void *x, int64_t x_stride, const void *gate,
                                int64_t gate_stride, const void *up, int64_t up_stride, const void *a, int64_t a_stride,
                                const void *b, int64_t b_stride, int64_t n, int64_t d, int64_t f, int activation, int type,
                                void *dx, int64_t dx_stride, void *dgate, int64_t dgate_stride, void *dup, int64_t dup_stride,
                                void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!layer_sizes_ok(n, d, f) || !act_ok(activation) || !type_ok(type)) return BHTSNE_EINVAL;
    if (!input_ok(dh, dh_stride, n, f, type) || !input_ok(x, x_stride, n, d, type) || !input_ok(a, a_stride, n, f, type)
        || !input_ok(b, b_stride, n, f, type))
        return BHTSNE_EINVAL;
    if (!output_ok(const_cast<void *>(gate), gate_stride, f, d, type) || !output_ok(const_cast<void *>(up), up_stride, f, d, type))
        return BHTSNE_EINVAL;
    if (!dx && !dgate && !dup) return BHTSNE_EINVAL;
    if ((dx && !output_ok(dx, dx_stride, n, d, type)) || (dgate && !output_ok(dgate, dgate_stride, f, d, type))
        || (dup && !output_ok(dup, dup_stride, f, d, type)))
        return BHTSNE_EINVAL;
    if (!apart({n > 0 ? dx : nullptr, dgate, dup}, {dh, x, gate, up, a, b})) return BHTSNE_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, bhtsne_gated_layer_workspace_size(n, d, f, type))) return BHTSNE_EWORKSPACE;
    GatedBackArgs g = {};
    g.dh = dh;
    g.dh_stride = dh_stride;
    g.x = x;
    g.x_stride = x_stride;
    g.gate = gate;
    g.gate_stride = gate_stride;
    g.up = up;
    g.up_stride = up_stride;
    g.a = a;
    g.a_stride = a_stride;
    g.b = b;
    g.b_stride = b_stride;
    g.n = n;
    g.d = d;
    g.f = f;
    g.act = Act(activation);
    g.type = Elem(type);
    g.dx = dx;
    g.dx_stride = dx_stride;
    g.dgate = dgate;
    g.dgate_stride = dgate_stride;
    g.dup = dup;
    g.dup_stride = dup_stride;
    g.ws = workspace;
    launch_gated_layer_backward(g, stream);
    return status();
}

int bhtsne_quantise_rows(const void *x, int64_t x_stride, int64_t n, int64_t d, int type, int8_t *q, int64_t q_stride,
                         float *scale, hipStream_t stream)
{
    if (n < 0 || n > kMost || d < 1 || d > kLinearMaxDepth || !type_ok(type)) return BHTSNE_EINVAL;
    if (!input_ok(x, x_stride, n, d, type) || !output_ok(q, q_stride, n, d, BHTSNE_I8)) return BHTSNE_EINVAL;
    if (!output_ok(scale, 1, n, 1, BHTSNE_F32)) return BHTSNE_EINVAL;
    if (n > 0 && !apart({q, scale}, {x})) return BHTSNE_EINVAL;
    QuantiseArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.q = q;
    a.q_stride = q_stride;
    a.scale = scale;
    a.n = n;
    a.d = d;
    a.type = Elem(type);
    launch_quantise_rows(a, stream);
    return status();
}

size_t bhtsne_linear_i8_workspace_size(int64_t n, int64_t d)
{
    if (n < 0 || n > kMost || d < 1 || d > kLinearMaxDepth) return 0;
    if (linear_few(n, d)) return 256; // none is needed
    const size_t depth = (size_t(d) + kLinearSlice - 1) / kLinearSlice * kLinearSlice;
    return (size_t(n) * 4 + 255) / 256 * 256 + (size_t(n) * depth + 255) / 256 * 256 + 256;
}

int bhtsne_linear_i8(const void *x, int64_t x_stride, int x_type, const float *x_scale, const int8_t *w, int64_t w_stride,
                     const float *w_scale, const void *bias, int64_t n, int64_t d, int64_t f, int type, int bias_type, void *out,
                     int64_t out_stride, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (n < 0 || n > kMost || d < 1 || d > kLinearMaxDepth || f < 1 || f > kLinearMaxFeatures) return BHTSNE_EINVAL;
    const bool whole = x_type == BHTSNE_I8;
    if (!type_ok(type) || (!whole && !type_ok(x_type)) || (bias_type != type && bias_type != BHTSNE_F32)) return BHTSNE_EINVAL;
    if (!input_ok(x, x_stride, n, d, x_type) || !output_ok(const_cast<int8_t *>(w), w_stride, f, d, BHTSNE_I8)) return BHTSNE_EINVAL;
    if (!output_ok(const_cast<float *>(w_scale), 1, f, 1, BHTSNE_F32) || !aligned(x_scale, BHTSNE_F32) || !aligned(bias, bias_type))
        return BHTSNE_EINVAL;
    if (whole ? !x_scale && n > 0 : x_scale != nullptr) return BHTSNE_EINVAL;
    if (!output_ok(out, out_stride, n, f, type)) return BHTSNE_EINVAL;
    if (n > 0 && !apart({out}, {x, x_scale, w, w_scale, bias})) return BHTSNE_EINVAL;
    LinearArgs a = {};
    a.w = w;
    a.w_stride = w_stride;
    a.w_scale = w_scale;
    a.bias = bias;
    a.n = n;
    a.d = d;
    a.f = f;
    a.out = out;
    a.out_stride = out_stride;
    a.type = Elem(type);
    a.bias_type = Elem(bias_type);
    if (whole) {
        a.x = static_cast<const int8_t *>(x);
        a.x_stride = x_stride;
        a.x_scale = x_scale;
    } else {
        if (!linear_few(n, d) && !workspace_ok(workspace, workspace_bytes, bhtsne_linear_i8_workspace_size(n, d))) return BHTSNE_EWORKSPACE;
        QuantiseArgs q = {};
        q.x = x;
        q.x_stride = x_stride;
        if (!linear_few(n, d)) {
            q.scale = static_cast<float *>(workspace);
            q.q = static_cast<int8_t *>(workspace) + (size_t(n) * 4 + 255) / 256 * 256;
        }
        q.q_stride = q.pad = (d + kLinearSlice - 1) / kLinearSlice * kLinearSlice;
        q.n = n;
        q.d = d;
        q.type = Elem(x_type);
        launch_linear_values(a, q, stream);
        return status();
    }
    launch_linear_i8(a, stream);
    return status();
}

size_t bhtsne_distil_loss_workspace_size(int64_t n, int64_t v)
{
    if (!distil_sizes_ok(n, v, 0)) return 0;
    const int parts = distil_parts(n, v);
    return 256 + (parts > 1 ? (size_t(n) * size_t(parts) * sizeof(float2) + 255) / 256 * 256 : 0); // 256: none is needed
}

int bhtsne_distil_loss_kept(const void *logits, int64_t stride, int64_t n, int64_t v, const int32_t *idx, int64_t idx_stride,
                            const void *teacher, int64_t teacher_stride, int64_t k, double temperature, int type, int teacher_type,
                            float *loss, float *lse, float *kept, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    DistilArgs a = {};
    if (!distil_inputs(&a, logits, stride, n, v, idx, idx_stride, teacher, teacher_stride, k, temperature, type, teacher_type))
        return BHTSNE_EINVAL;
    if ((!loss && !lse && !kept && n > 0) || !aligned(loss, BHTSNE_F32) || !aligned(lse, BHTSNE_F32) || !aligned(kept, BHTSNE_F32))
        return BHTSNE_EINVAL;
    if (a.parts > 1 && !workspace_ok(workspace, workspace_bytes, bhtsne_distil_loss_workspace_size(n, v))) return BHTSNE_EWORKSPACE;
    if (n > 0 && !apart({loss, lse, kept}, {logits, k > 0 ? idx : nullptr, k > 0 ? teacher : nullptr, a.parts > 1 ? workspace : nullptr}))
        return BHTSNE_EINVAL;
    a.loss = loss;
    a.lse = lse;
    a.kept = kept;
    a.part = static_cast<float2 *>(workspace);
    launch_distil_loss(a, stream);
    return status();
}

int bhtsne_distil_loss(const void *logits, int64_t stride, int64_t n, int64_t v, const int32_t *idx, int64_t idx_stride,
                       const void *teacher, int64_t teacher_stride, int64_t k, double temperature, int type, int teacher_type,
                       float *loss, float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!loss && !lse && n > 0) return BHTSNE_EINVAL;
    return bhtsne_distil_loss_kept(logits, stride, n, v, idx, idx_stride, teacher, teacher_stride, k, temperature, type, teacher_type,
                                   loss, lse, nullptr, workspace, workspace_bytes, stream);
}

int bhtsne_distil_loss_backward_kept(const float *dloss, const void *logits, int64_t stride, int64_t n, int64_t v, const int32_t *idx,
                                     int64_t idx_stride, const void *teacher, int64_t teacher_stride, int64_t k, const float *lse,
                                     const float *kept, double temperature, int type, int teacher_type, void *dlogits,
                                     int64_t dlogits_stride, hipStream_t stream)
{
    DistilArgs a = {};
    if (!distil_inputs(&a, logits, stride, n, v, idx, idx_stride, teacher, teacher_stride, k, temperature, type, teacher_type))
        return BHTSNE_EINVAL;
    if (((!dloss || !lse) && n > 0) || !aligned(dloss, BHTSNE_F32) || !aligned(lse, BHTSNE_F32) || !aligned(kept, BHTSNE_F32))
        return BHTSNE_EINVAL;
    if (!output_ok(dlogits, dlogits_stride, n, v, type)) return BHTSNE_EINVAL;
    if (n > 0 && !apart({dlogits}, {dloss, lse, kept, k > 0 ? idx : nullptr, k > 0 ? teacher : nullptr})) return BHTSNE_EINVAL;
    // over the logits, row by row: with another stride a row would be written where another is still to be read
    if (n > 1 && dlogits == logits && dlogits_stride != stride) return BHTSNE_EINVAL;
    a.dloss = dloss;
    a.lse_in = lse;
    a.kept_in = kept;
    a.out = dlogits;
    a.out_stride = dlogits_stride;
    launch_distil_loss_backward(a, stream);
    return status();
}

int bhtsne_distil_loss_backward(const float *dloss, const void *logits, int64_t stride, int64_t n, int64_t v, const int32_t *idx,
                                int64_t idx_stride, const void *teacher, int64_t teacher_stride, int64_t k, const float *lse,
                                double temperature, int type, int teacher_type, void *dlogits, int64_t dlogits_stride,
                                hipStream_t stream)
{
    return bhtsne_distil_loss_backward_kept(dloss, logits, stride, n, v, idx, idx_stride, teacher, teacher_stride, k, lse, nullptr,
                                            temperature, type, teacher_type, dlogits, dlogits_stride, stream);
}

} // extern "C"
