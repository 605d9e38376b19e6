// Products of 8-bit integers with a scale for each point and each feature.
//
//   quantise:  s = max|x| / 127 (fp32),  q = x / s rounded to the nearest integer, ties to even
//   product:   out = s_i t_j sum_k q_ik w_jk + bias_j
//
// The sums are exact: 32-bit integers hold 131071 products of 8-bit values.  The
// quantisation reads a row once, into the registers of a wave or a block: 70001 x
// 2000 bf16, 422 MB, 93 to 104 us (4.5 TB/s), bound by HBM and by the vector
// instructions, which are issued in 98 % of that time.  The product runs on the matrix
// cores' 8-bit instructions: 70001 x 2000 to 2000, 0.56 TOP, 310 us, nine rounds of
// CUs of which each ends with outputs that nothing covers.
#include "products.hpp"

namespace bht {
namespace {

using namespace prod;

// ------------------------------------------------------------------ quantisation
constexpr int kRowValues = 16; // of a thread at a time

// 16 values of a row of d from `at` on, zeros behind its end
template <typename E> __device__ inline void load_values(const E *row, int64_t at, int64_t d, float (&v)[kRowValues])
{
    constexpr int kV = 16 / int(sizeof(E));
#pragma unroll
    for (int h = 0; h < kRowValues / kV; ++h) {
        const Piece x = any_piece<E>(reinterpret_cast<const char *>(row), (at + h * kV) * int64_t(sizeof(E)), d * int64_t(sizeof(E)));
        E e[kV];
        __builtin_memcpy(e, &x, 16);
#pragma unroll
        for (int k = 0; k < kV; ++k) v[h * kV + k] = float(e[k]);
    }
}

// x / s rounded as the quotient in 64 bits is.  The product with 1 / s is off by some 2e-5 at most: nearer to the border
// of two integers (and where 1 / s is infinite) the division decides, which is exact there.
__device__ inline int quantise(float x, float s, float inverse)
{
    const float r = x * inverse, k = rintf(r);
    int q = int(k);
    if (!(fabsf(r - k) < 0.4999f)) {
        const double d = rint(double(x) / double(s));
        q = int(fmin(fmax(d, -127.0), 127.0)); // a scale among the smallest numbers is a rough one
    }
    return q;
}

template <typename E, int kThreads> __global__ __launch_bounds__(kThreads) void quantise_kernel(QuantiseArgs a)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ float s_max[kWaves];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E *x = static_cast<const E *>(a.x) + row * a.x_stride;
        int8_t *q = a.q + row * a.q_stride;
        float v[kRowValues], top = 0.0f;
        const auto take = [&](int64_t at) {
            load_values(x, at, a.d, v);
#pragma unroll
            for (int e = 0; e < kRowValues; ++e) {
                const float m = fabsf(v[e]);
                top = m <= top ? top : m < INFINITY ? m : INFINITY; // NaN counts as an infinity, which stays
            }
        };
#pragma unroll
        for (int e = 0; e < kRowValues; ++e) v[e] = 0.0f; // behind the row's end
        for (int64_t at = int64_t(threadIdx.x) * kRowValues; at < a.d; at += kThreads * kRowValues) take(at);
        top = wave_max(top);
        if constexpr (kWaves > 1) {
            if (lane_id() == 0) s_max[threadIdx.x / kWave] = top;
            __syncthreads();
            top = s_max[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_max[w]);
            __syncthreads();
        }
        const bool finite = top < INFINITY;
        const float scale = finite ? top / 127.0f : NAN, inverse = 1.0f / scale;
        if (threadIdx.x == 0) a.scale[row] = scale;
        const bool aligned = (reinterpret_cast<uintptr_t>(q) & 15) == 0;
        const int64_t width = a.pad > a.d ? a.pad : a.d;
        for (int64_t at = int64_t(threadIdx.x) * kRowValues; at < width; at += kThreads * kRowValues) {
            if (width > kThreads * kRowValues) load_values(x, at, a.d, v);
            struct alignas(16) {
                int8_t v[kRowValues];
            } out;
#pragma unroll
            for (int e = 0; e < kRowValues; ++e) out.v[e] = int8_t(finite && scale > 0.0f ? quantise(v[e], scale, inverse) : 0);
            if (aligned && at + kRowValues <= width) {
                *reinterpret_cast<Piece *>(q + at) = __builtin_bit_cast(Piece, out);
            } else {
#pragma unroll
                for (int e = 0; e < kRowValues; ++e)
                    if (at + e < width) q[at + e] = out.v[e];
            }
        }
    }
}

template <typename E> void run_quantise(const QuantiseArgs &a, hipStream_t st)
{
    const uint32_t blocks = uint32_t(a.n < (int64_t(1) << 20) ? a.n : int64_t(1) << 20);
    if (a.d <= 64 * kRowValues)
        quantise_kernel<E, 64><<<blocks, 64, 0, st>>>(a);
    else if (a.d <= 128 * kRowValues)
        quantise_kernel<E, 128><<<blocks, 128, 0, st>>>(a);
    else if (a.d <= 256 * kRowValues)
        quantise_kernel<E, 256><<<blocks, 256, 0, st>>>(a);
    else
        quantise_kernel<E, 1024><<<blocks, 1024, 0, st>>>(a);
}

// ------------------------------------------------------------------ product
struct LinearOut {
    const float *x_scale, *w_scale;
    const void *bias;
    void *out;
    int64_t stride;
    bool wide_bias, vec, inner;
};

template <typename E, typename T, bool kAny, Tail kTail>
__global__ __launch_bounds__(T::kThreads) void linear8_kernel(Product p, LinearOut o)
{
    constexpr int kRun = T::kJ;
    each_tile<int8_t, T, Form::kRows, kAny, kTail>(p, [&](int32_t bi, int32_t bj, Ops<int8_t>::Acc (&acc)[T::kI][T::kJ]) {
        if (o.inner && tile_inside<T, Form::kRows>(p, bi, bj)) {
            const InnerRuns<T, Form::kRows> runs(bi, bj);
            const auto to = runs.template to<E>(o.out, o.stride);
            float scale[kRun], bias[kRun];
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                const int64_t at = runs.feature + runs.lane_feature + e;
                scale[e] = o.w_scale[at];
                bias[e] = !o.bias ? 0.0f : o.wide_bias ? static_cast<const float *>(o.bias)[at] : float(static_cast<const E *>(o.bias)[at]);
            }
#pragma unroll
            for (int i = 0; i < T::kI; ++i) {
                float s[4]; // before the stores, which a load behind them waits for (one by one: 416 us a call for 400)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = (o.x_scale + runs.row + (16 * i + r))[runs.lane_row];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v[kRun];
#pragma unroll
                    for (int e = 0; e < kRun; ++e) v[e] = float(acc[i][e][r]) * s[r] * scale[e] + bias[e];
                    to.put(i, r, v);
                }
            }
            return;
        }
        float scale[kRun], bias[kRun];
        each_run<T, Form::kRows>(bi, bj, [&](int64_t point, int64_t feature, int i, int r) {
            if (i == 0 && r == 0) {
#pragma unroll
                for (int e = 0; e < kRun; ++e) {
                    const int64_t at = feature + e < p.features ? feature + e : p.features - 1;
                    scale[e] = o.w_scale[at];
                    bias[e] = 0.0f;
                }
            }
            if (i == 0 && r == 0 && o.bias) {
                if (o.wide_bias) {
#pragma unroll
                    for (int e = 0; e < kRun; ++e) bias[e] = static_cast<const float *>(o.bias)[feature + e < p.features ? feature + e : p.features - 1];
                } else {
#pragma unroll
                    for (int e = 0; e < kRun; ++e) bias[e] = float(static_cast<const E *>(o.bias)[feature + e < p.features ? feature + e : p.features - 1]);
                }
            }
            if (point >= p.rows) return;
            const float s = o.x_scale[point];
            float v[kRun];
#pragma unroll
            for (int e = 0; e < kRun; ++e) v[e] = float(acc[i][e][r]) * s * scale[e] + bias[e];
            store_run(static_cast<E *>(o.out) + point * o.stride + feature, v, p.features - feature, o.vec);
        });
    });
}

template <typename E, typename T, bool kAny, Tail kTail = Tail::kWhole> void run_linear(const LinearArgs &a, hipStream_t st)
{
    Product p = {};
    p.B = reinterpret_cast<const char *>(a.w);
    p.a_stride = a.x_stride;
    p.b_stride = a.w_stride;
    p.features = a.f;
    p.bytes = a.d;
    p.slices = p.per_split = int32_t((a.d + kSlice - 1) / kSlice);
    p.across = int32_t((a.f + T::kN - 1) / T::kN);
    const size_t lds = size_t(kAny && p.slices == 1 ? 1 : T::kStages) * T::kBuffer;
    const int64_t most = kMostTiles / p.across > 0 ? kMostTiles / p.across * T::kM : T::kM;
    for (int64_t from = 0; from < a.n; from += most) {
        p.A = reinterpret_cast<const char *>(a.x) + from * a.x_stride;
        p.rows = a.n - from < most ? a.n - from : most;
        p.down = int32_t((p.rows + T::kM - 1) / T::kM);
        LinearOut o = {};
        o.x_scale = a.x_scale + from;
        o.w_scale = a.w_scale;
        o.bias = a.bias;
        o.out = static_cast<E *>(a.out) + from * a.out_stride;
        o.stride = a.out_stride;
        o.wide_bias = a.bias_type == Elem::kF32;
        o.inner = runs_inner<E, T::kJ>(a.out, a.out_stride);
        o.vec = runs_aligned<E, T::kJ>(a.out, a.out_stride);
        linear8_kernel<E, T, kAny, kTail><<<blocks_of<T>(uint32_t(p.down) * uint32_t(p.across)), T::kThreads, lds, st>>>(p, o);
    }
}

// A few points (few_points).  X: their type; int8 as they are, else the block quantises them into LDS while its weights are
// under way to it: one launch (1 x 2048 to 8192 bf16 8.4 us, of which a launch is 2.5; by two 12 and the gap between them).
template <typename E, typename X, int kI>
__global__ __launch_bounds__(kFewWaves *kWave) void linear8_few_kernel(Product p, LinearOut o)
{
    constexpr bool kWhole = sizeof(X) == 1;
    constexpr int kThreads = kFewWaves * kWave;
    static_assert(kWhole || kI == 1, "few points are quantised");
    __shared__ int32_t s_sum[kFewWaves][1][kI][256];
    __shared__ float s_scale[kFewPoints], s_max[kFewWaves];
    __shared__ __align__(16) int8_t s_x[kWhole ? 16 : kFewValues];
    const int64_t feature = int64_t(blockIdx.x) * 16, first = int64_t(blockIdx.y) * (16 * kI);
    const int lane = lane_id(), point_row = lane % 16 < p.rows ? lane % 16 : int(p.rows) - 1;
    const int32_t width = p.slices * kSlice;
    const auto quantise_all = [&] {
        if constexpr (kWhole) return;
        for (int r = 0; r < int(p.rows); ++r) {
            const X *x = reinterpret_cast<const X *>(p.A + r * p.a_stride);
            float v[kRowValues], top = 0.0f;
#pragma unroll
            for (int e = 0; e < kRowValues; ++e) v[e] = 0.0f;
            const int at = int(threadIdx.x) * kRowValues; // the whole row at once
            static_assert(kFewValues <= kThreads * kRowValues, "a row is in the threads' registers");
            if (at < p.bytes) load_values(x, at, p.bytes, v);
#pragma unroll
            for (int e = 0; e < kRowValues; ++e) {
                const float m = fabsf(v[e]);
                top = m <= top ? top : m < INFINITY ? m : INFINITY;
            }
            top = wave_max(top);
            if (lane == 0) s_max[threadIdx.x / kWave] = top;
            __syncthreads();
            top = s_max[0];
#pragma unroll
            for (int k = 1; k < kFewWaves; ++k) top = fmaxf(top, s_max[k]);
            const bool finite = top < INFINITY;
            const float scale = finite ? top / 127.0f : NAN, inverse = 1.0f / scale;
            if (threadIdx.x == 0) s_scale[r] = scale;
            if (at < width) {
                struct alignas(16) {
                    int8_t v[kRowValues];
                } q;
#pragma unroll
                for (int e = 0; e < kRowValues; ++e) q.v[e] = int8_t(finite && scale > 0.0f ? quantise(v[e], scale, inverse) : 0);
                *reinterpret_cast<Piece *>(s_x + r * width + at) = __builtin_bit_cast(Piece, q);
            }
            __syncthreads();
        }
    };
    const char *row[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const int64_t point = first + 16 * i + lane % 16;
        row[i] = p.A + (point < p.rows ? point : p.rows - 1) * p.a_stride;
    }
    const auto x = [&](int32_t slice, int half, int i) {
        const int64_t k = int64_t(slice) * kSlice + half * 64 + lane / 16 * 16;
        if constexpr (kWhole)
            return int64_t(slice + 1) * kSlice <= p.bytes ? inner_piece(row[i] + k) : any_piece<int8_t>(row[i], k, p.bytes);
        else
            return *reinterpret_cast<const Piece *>(s_x + point_row * width + k);
    };
    Ops<int8_t>::Acc acc[1][kI] = {};
    few_points<int8_t, 1, kI>(p, feature, quantise_all, x, acc);
    few_put(acc, s_sum);
    for (int t = int(threadIdx.x); t < 256 * kI; t += kThreads) {
        const int64_t point = first + t / 16, at = feature + t % 16, held = at < p.features ? at : p.features - 1;
        float bias = 0.0f;
        if (o.bias) bias = o.wide_bias ? static_cast<const float *>(o.bias)[held] : float(static_cast<const E *>(o.bias)[held]);
        if (point >= p.rows || at >= p.features) continue;
        const float s = kWhole ? o.x_scale[point] : s_scale[t / 16 % kFewPoints];
        static_cast<E *>(o.out)[point * o.stride + at] = rounded<E>(float(few_sum(s_sum, 0, t / 256, t % 256)) * s * o.w_scale[at] + bias);
    }
}

template <typename E, typename X, int kI> void run_linear_few(const LinearArgs &a, const void *x, int64_t x_stride, hipStream_t st)
{
    Product p = {};
    p.A = static_cast<const char *>(x);
    p.B = reinterpret_cast<const char *>(a.w);
    p.a_stride = x_stride * int64_t(sizeof(X));
    p.b_stride = a.w_stride;
    p.rows = a.n;
    p.features = a.f;
    p.bytes = a.d;
    p.slices = p.per_split = int32_t(slices_of(a.d));
    LinearOut o = {};
    o.x_scale = a.x_scale;
    o.w_scale = a.w_scale;
    o.bias = a.bias;
    o.out = a.out;
    o.stride = a.out_stride;
    o.wide_bias = a.bias_type == Elem::kF32;
    const dim3 grid(uint32_t((a.f + 15) / 16), uint32_t((a.n + 16 * kI - 1) / (16 * kI)));
    linear8_few_kernel<E, X, kI><<<grid, kFewWaves * kWave, 0, st>>>(p, o);
}

template <typename E> bool few_and_quantised(const LinearArgs &a, const QuantiseArgs &q, hipStream_t st)
{
    if (!linear_few(a.n, a.d)) return false;
    if (q.type == Elem::kF32)
        run_linear_few<E, float, 1>(a, q.x, q.x_stride, st);
    else if (q.type == Elem::kF16)
        run_linear_few<E, f16, 1>(a, q.x, q.x_stride, st);
    else
        run_linear_few<E, bf16, 1>(a, q.x, q.x_stride, st);
    return true;
}

template <typename E> void run_linear_type(const LinearArgs &a, hipStream_t st)
{
    if (a.n <= kFewPoints) return run_linear_few<E, int8_t, 1>(a, a.x, a.x_stride, st);
    const bool any = !aligned16(a.x, a.x_stride) || !aligned16(a.w, a.w_stride) || a.d % 16 != 0;
    if (few_tiles(a.n, a.f, !any)) return run_linear_few<E, int8_t, kFewRows / 16>(a, a.x, a.x_stride, st);
    const Side side = plan_product(a.n, a.f, slices_of(a.d), false, false,
                                   any || a.x_stride > kLargeStride || a.w_stride > kLargeStride ? Side::kMiddle : Side::kLarge).side;
    if (any) {
        if (side == Side::kMiddle) return run_linear<E, TileMiddle, true>(a, st);
        return run_linear<E, TileSmall, true>(a, st);
    }
    if (side == Side::kLarge) {
        if (a.d % kSlice == 0) return run_linear<E, TileLarge, false, Tail::kWhole>(a, st);
        return a.padded ? run_linear<E, TileLarge, false, Tail::kFirst>(a, st) : run_linear<E, TileLarge, false, Tail::kZeros>(a, st);
    }
    if (side == Side::kMiddle) return run_linear<E, TileMiddle, false>(a, st);
    run_linear<E, TileSmall, false>(a, st);
}

} // namespace

void launch_quantise_rows(const QuantiseArgs &a, hipStream_t st)
{
    if (a.n == 0) return;
    if (a.type == Elem::kF32) return run_quantise<float>(a, st);
    if (a.type == Elem::kF16) return run_quantise<f16>(a, st);
    run_quantise<bf16>(a, st);
}

void launch_linear_i8(const LinearArgs &a, hipStream_t st)
{
    if (a.n == 0) return;
    if (a.type == Elem::kF32) return run_linear_type<float>(a, st);
    if (a.type == Elem::kF16) return run_linear_type<f16>(a, st);
    run_linear_type<bf16>(a, st);
}

void launch_linear_values(LinearArgs a, const QuantiseArgs &q, hipStream_t st)
{
    if (a.n == 0) return;
    const bool done = a.type == Elem::kF32 ? few_and_quantised<float>(a, q, st) : a.type == Elem::kF16 ? few_and_quantised<f16>(a, q, st) : few_and_quantised<bf16>(a, q, st);
    if (done) return;
    launch_quantise_rows(q, st);
    a.x = q.q;
    a.x_stride = q.q_stride;
    a.x_scale = q.scale;
    a.padded = true;
    launch_linear_i8(a, st);
}

} // namespace bht
