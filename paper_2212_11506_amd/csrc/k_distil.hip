// The loss of a row of logits z over v classes (points, landmarks) against a
// teacher's logits u of k listed ones, and its gradient:
//
//   t = softmax(u / T) over the list,  q = softmax(z / T) over all,  lse = log sum exp(z / T)
//   loss = sum_j t_j (log t_j - z_idx(j) / T + lse)
//   dz   = dloss / T (q - t at the listed places)
//
// A row's logits are read once: forward with the running maximum and sum of a
// softmax in each lane, joined over the lanes and, where few rows are shared out
// over several blocks, over the parts by a second launch.  Backward reads and
// writes each once, four operations and an exponential a value.  HBM bounds both:
// 4096 x 70001 bf16 105 us forward (5.5 TB/s), 2048 x 70000 124 backward (4.6).
// Maximum and sum of a lane are fp32, the joined sum and the list's terms fp64; the
// only rounding to fewer bits is that of dz.  A lane adds its terms one after another:
// v / 64 of a wave's row (32 at most), a 256th of a block's row or part.  Rows are in
// 2048 / n parts, of 8192 values or more, so from 1025 rows on in one: 274 terms of
// 70001 values, 5078 of 1.3M, whose roundings are 2^-24 of the sum each at most.
#include <type_traits>

#include "dense.hpp"

namespace bht {
namespace {

constexpr double kLog2e = 1.4426950408889634;

template <typename E> struct alignas(16) Vec {
    static constexpr int kV = 16 / int(sizeof(E));
    E v[kV];
};

// 16 bytes at the values' own alignment; and 16 aligned ones, which leave no lines in the caches (2048 x 70000 bf16, 573 MB
// read and written: 141 us without, 125 so; 16 x 1.3M fp16 19.6 and 19.1; loads that leave none 137)
template <typename E> __device__ inline Vec<E> load_vec(const E *p)
{
    Vec<E> v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
template <typename E> __device__ inline void store_vec(E *p, const Vec<E> &v)
{
    __builtin_nontemporal_store(__builtin_bit_cast(uint4v, v), reinterpret_cast<uint4v *>(p));
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The running maximum m and sum of exp2((z - m) c) of a lane's logits.  Logits of minus infinity count nothing; NaN and
// plus infinity make the sum NaN, as in the formula.
struct Running {
    float m, s;
    template <int N> __device__ void add(const float (&z)[N], float c)
    {
        float top = z[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
        top = fmaxf(m, top);
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = s * exp2_fast((m - base) * c);
#pragma unroll
        for (int e = 0; e < N; ++e) sum += exp2_fast((z[e] - base) * c);
        m = top;
        s = sum;
    }
};

// Joins the lanes of a block: every thread has the maximum and the sum.
template <int kThreads> __device__ inline void join(float &m, double &s, float lane_sum, float c, double *s_sum, float *s_max)
{
    constexpr int kWaves = kThreads / kWave;
    float top = wave_max(m);
    if constexpr (kWaves > 1) {
        if (lane_id() == 0) s_max[threadIdx.x / kWave] = top;
        __syncthreads();
        top = s_max[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_max[w]);
    }
    const float base = top == -INFINITY ? 0.0f : top;
    double sum = wave_sum(double(lane_sum) * double(exp2_fast((m - base) * c)));
    if constexpr (kWaves > 1) {
        if (lane_id() == 0) s_sum[threadIdx.x / kWave] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += s_sum[w];
        __syncthreads(); // both arrays are written again
    }
    m = top;
    s = sum;
}

template <int kThreads> __device__ inline double block_sum(double v, double *s_sum)
{
    constexpr int kWaves = kThreads / kWave;
    v = wave_sum(v);
    if constexpr (kWaves > 1) {
        if (lane_id() == 0) s_sum[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += s_sum[w];
        __syncthreads();
    }
    return v;
}

// The teacher's softmax over a row's list: the largest u of a class that exists, and the sum of exp((u - top) / T).
// Entries whose index is no class are absent.  A list without entries has the sum 0, and no other has: the largest u adds 1
// (NaN leaves no trace in the top, but makes the sum NaN).
struct List {
    float top;
    double sum;
    __device__ inline bool empty() const { return sum == 0.0; }
};
template <typename TE, int kThreads>
__device__ inline List list_of(const DistilArgs &a, int64_t row, float c, double *s_sum, float *s_max)
{
    const int32_t *idx = a.idx + row * a.idx_stride;
    const TE *u = static_cast<const TE *>(a.teacher) + row * a.teacher_stride;
    Running r{-INFINITY, 0.0f};
    for (int j = threadIdx.x; j < a.k; j += kThreads) {
        const bool there = uint32_t(idx[j]) < uint64_t(a.v);
        const float x[1] = {there ? float(u[j]) : -INFINITY};
        r.add(x, c);
    }
    List l;
    l.top = r.m;
    join<kThreads>(l.top, l.sum, r.s, c, s_sum, s_max);
    return l;
}

// Logits [from, to) of a row through a lane's running sum: single values up to the first 16-byte boundary, vectors, rest.
// (Vectors at any alignment, whose sums would not depend on it: 4096 x 70001 bf16 133 us, so 112.)
template <typename E, int kThreads>
__device__ inline Running run_over(const E *row, int64_t from, int64_t to, float c)
{
    constexpr int kV = Vec<E>::kV, kAtOnce = 4;
    Running r{-INFINITY, 0.0f};
    const E *p = row + from;
    const int64_t count = to - from;
    int64_t head = int64_t((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / int64_t(sizeof(E));
    if (head > count) head = count;
    if (int64_t(threadIdx.x) < head) {
        const float x[1] = {float(p[threadIdx.x])};
        r.add(x, c);
    }
    p += head;
    const int64_t vectors = (count - head) / kV;
    const Vec<E> *q = reinterpret_cast<const Vec<E> *>(p);
    int64_t i = threadIdx.x;
    for (; i + (kAtOnce - 1) * kThreads < vectors; i += kAtOnce * kThreads) {
        Vec<E> x[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) x[u] = q[i + u * kThreads];
        float z[kAtOnce * kV];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int e = 0; e < kV; ++e) z[u * kV + e] = float(x[u].v[e]);
        r.add(z, c);
    }
    for (; i < vectors; i += kThreads) {
        const Vec<E> x = q[i];
        float z[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) z[e] = float(x.v[e]);
        r.add(z, c);
    }
    const int64_t rest = head + vectors * kV;
    if (rest + int64_t(threadIdx.x) < count) {
        const float x[1] = {float(p[vectors * kV + threadIdx.x])};
        r.add(x, c);
    }
    return r;
}

// Values [from, to) of part `part` of a row: whole vectors of the widest type, so that parts start alike
__device__ inline void part_of(const DistilArgs &a, int part, int64_t &from, int64_t &to)
{
    const int64_t each = ((a.v + a.parts - 1) / a.parts + 7) / 8 * 8;
    from = part * each < a.v ? part * each : a.v;
    to = from + each < a.v ? from + each : a.v;
}

// The row's outputs from its maximum and sum.  The loss takes a listed logit's distance from the maximum before anything is
// added to it: next to logits as large as the type's lowest value, for classes that are masked out, the sum's logarithm vanishes.
template <typename E, typename TE, int kThreads>
__device__ inline void finish(const DistilArgs &a, int64_t row, float m, double s, float c, double *s_sum, float *s_max)
{
    const double log_s = log(s);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = float(double(m) / a.temperature + log_s);
        if (a.kept) {
            a.kept[2 * row] = m;
            a.kept[2 * row + 1] = float(s);
        }
    }
    if (!a.loss) return;
    const List l = list_of<TE, kThreads>(a, row, c, s_sum, s_max);
    const E *z = static_cast<const E *>(a.logits) + row * a.stride;
    const int32_t *idx = a.idx + row * a.idx_stride;
    const TE *u = static_cast<const TE *>(a.teacher) + row * a.teacher_stride;
    const double log_sum = log(l.sum);
    double sum = 0.0;
    for (int j = threadIdx.x; j < a.k; j += kThreads) {
        const int32_t at = idx[j];
        const bool there = uint32_t(at) < uint64_t(a.v);
        const float above = (there ? float(u[j]) : -INFINITY) - l.top; // NaN where the list is empty
        const double t = double(exp2_fast(above * c)) / l.sum;
        const double zj = double(float(z[there ? at : 0]));
        const double term = t * (double(above) / a.temperature - log_sum + (double(m) - zj) / a.temperature + log_s);
        sum += l.empty() || t == 0.0 ? 0.0 : term;
    }
    sum = block_sum<kThreads>(sum, s_sum);
    if (threadIdx.x == 0) a.loss[row] = float(sum);
}

// One part of a row a block; rows of one part are finished at once.
template <typename E, typename TE, int kThreads>
__global__ __launch_bounds__(kThreads) void distil_kernel(DistilArgs a)
{
    __shared__ double s_sum[kThreads / kWave];
    __shared__ float s_max[kThreads / kWave];
    const float c = float(kLog2e / a.temperature);
    const int64_t items = a.n * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const int part = int(item - row * a.parts);
        int64_t from, to;
        part_of(a, part, from, to);
        const Running r = run_over<E, kThreads>(static_cast<const E *>(a.logits) + row * a.stride, from, to, c);
        float m = r.m;
        double s;
        join<kThreads>(m, s, r.s, c, s_sum, s_max);
        if (a.parts > 1) {
            if (threadIdx.x == 0) a.part[item] = make_float2(m, float(s));
        } else {
            finish<E, TE, kThreads>(a, row, m, s, c, s_sum, s_max);
        }
    }
}

// Rows of several parts: a wave joins them
template <typename E, typename TE> __global__ __launch_bounds__(kWave) void distil_join_kernel(DistilArgs a)
{
    const float c = float(kLog2e / a.temperature);
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        Running r{-INFINITY, 0.0f};
        for (int p = threadIdx.x; p < a.parts; p += kWave) {
            const float2 v = a.part[row * a.parts + p];
            const float top = fmaxf(r.m, v.x), base = top == -INFINITY ? 0.0f : top;
            r.s = r.s * exp2_fast((r.m - base) * c) + v.y * exp2_fast((v.x - base) * c);
            r.m = top;
        }
        float m = r.m;
        double s;
        join<kWave>(m, s, r.s, c, nullptr, nullptr);
        finish<E, TE, kWave>(a, row, m, s, c, nullptr, nullptr);
    }
}

// One part of a row a block.  dz may be written over the logits, so the listed ones of the part are read before, and their
// values written behind the others.  A class that is listed more than once is summed up by its first entry, in the list's order.
template <typename E, typename TE, int kThreads>
__global__ __launch_bounds__(kThreads) void distil_back_kernel(DistilArgs a)
{
    __shared__ double s_sum[kThreads / kWave];
    __shared__ float s_max[kThreads / kWave];
    extern __shared__ __align__(16) char s_mem[];
    int32_t *s_at = reinterpret_cast<int32_t *>(s_mem); // class, -1 without one
    float *s_t = reinterpret_cast<float *>(s_at + a.k); // its share of the teacher
    float *s_v = s_t + a.k;                             // dz there
    int32_t *s_first = reinterpret_cast<int32_t *>(s_v + a.k); // whether this entry writes it
    constexpr int kV = Vec<E>::kV;
    const float c = float(kLog2e / a.temperature);
    const int64_t items = a.n * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        int64_t from, to;
        part_of(a, int(item - row * a.parts), from, to);
        const E *z = static_cast<const E *>(a.logits) + row * a.stride;
        E *out = static_cast<E *>(a.out) + row * a.out_stride;
        const List l = list_of<TE, kThreads>(a, row, c, s_sum, s_max);
        const bool empty = l.empty();
        // q = exp2((z - high) c) factor: from the row's largest logit and its sum, which lose nothing; or with lse T as a high
        // and a low part, where lse's rounding makes q off by |lse| 2^-24
        const float given = a.lse_in[row];
        const double g = double(a.dloss[row]) / a.temperature, lse = double(given) * a.temperature;
        float high = float(lse), factor;
        if (a.kept_in && !(fabsf(given) < kDistilNear)) {
            high = a.kept_in[2 * row];
            factor = float(g / double(a.kept_in[2 * row + 1]));
        } else {
            const float low = high == high && fabsf(high) < INFINITY ? float(lse - double(high)) : 0.0f;
            factor = float(g) * exp2_fast(-low * c);
        }
        const int32_t *idx = a.idx + row * a.idx_stride;
        const TE *u = static_cast<const TE *>(a.teacher) + row * a.teacher_stride;
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            const int32_t at = idx[j];
            const bool there = uint32_t(at) < uint64_t(a.v);
            const float t = float(double(exp2_fast(((there ? float(u[j]) : -INFINITY) - l.top) * c)) / l.sum);
            s_at[j] = there && !empty ? at : -1;
            s_t[j] = t;
        }
        __syncthreads();
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            const int32_t at = s_at[j];
            if (at < from || at >= to) continue;
            double t = 0.0;
            bool first = true;
            for (int i = 0; i < a.k; ++i) {
                if (s_at[i] != at) continue;
                if (i < j) first = false;
                t += double(s_t[i]);
            }
            s_v[j] = float(double(factor) * double(exp2_fast((float(z[at]) - high) * c)) - g * t);
            s_first[j] = first;
        }
        __syncthreads();
        const auto dense = [&](float x) { return E(empty ? 0.0f : factor * exp2_fast((x - high) * c)); };
        const E *p = z + from;
        E *o = out + from;
        const int64_t count = to - from;
        // single values up to the output's first 16-byte boundary, vectors, rest; the logits at whatever alignment they have
        int64_t head = int64_t((16 - (reinterpret_cast<uintptr_t>(o) & 15)) & 15) / int64_t(sizeof(E));
        if (head > count) head = count;
        if (int64_t(threadIdx.x) < head) o[threadIdx.x] = dense(float(p[threadIdx.x]));
        p += head;
        o += head;
        const int64_t vectors = (count - head) / kV;
        constexpr int kAtOnce = 4;
        int64_t i = threadIdx.x;
        for (; i + (kAtOnce - 1) * kThreads < vectors; i += kAtOnce * kThreads) {
            Vec<E> x[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) x[u] = load_vec(p + (i + u * kThreads) * kV);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
#pragma unroll
                for (int e = 0; e < kV; ++e) x[u].v[e] = dense(float(x[u].v[e]));
                store_vec(o + (i + u * kThreads) * kV, x[u]);
            }
        }
        for (; i < vectors; i += kThreads) {
            Vec<E> x = load_vec(p + i * kV);
#pragma unroll
            for (int e = 0; e < kV; ++e) x.v[e] = dense(float(x.v[e]));
            store_vec(o + i * kV, x);
        }
        const int64_t rest = vectors * kV + threadIdx.x;
        if (rest < count - head) o[rest] = dense(float(p[rest]));
        __syncthreads();
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            const int32_t at = s_at[j];
            if (at >= from && at < to && s_first[j]) out[at] = E(s_v[j]);
        }
        __syncthreads();
    }
}

constexpr int64_t kMostBlocks = int64_t(1) << 22; // a block takes more than one part beyond

int blocks_of(int64_t items) { return int(items < kMostBlocks ? items : kMostBlocks); }

template <typename E, typename TE> void launch_forward(const DistilArgs &a, hipStream_t st)
{
    const int64_t items = a.n * a.parts;
    if (a.v <= kDistilWave)
        distil_kernel<E, TE, kWave><<<blocks_of(items), kWave, 0, st>>>(a);
    else
        distil_kernel<E, TE, 256><<<blocks_of(items), 256, 0, st>>>(a);
    if (a.parts > 1) distil_join_kernel<E, TE><<<blocks_of(a.n), kWave, 0, st>>>(a);
}

template <typename E, typename TE> void launch_backward(const DistilArgs &a, hipStream_t st)
{
    const int64_t items = a.n * a.parts;
    const size_t lds = size_t(a.k) * 16;
    if (a.v <= kDistilWave)
        distil_back_kernel<E, TE, kWave><<<blocks_of(items), kWave, lds, st>>>(a);
    else
        distil_back_kernel<E, TE, 256><<<blocks_of(items), 256, lds, st>>>(a);
}

template <typename F> void with_types(const DistilArgs &a, F f)
{
    if (a.type == Elem::kF32) return f(float(), float());
    if (a.type == Elem::kF16) return a.wide_teacher ? f(f16(), float()) : f(f16(), f16());
    return a.wide_teacher ? f(bf16(), float()) : f(bf16(), bf16());
}

} // namespace

void launch_distil_loss(const DistilArgs &a, hipStream_t st)
{
    if (a.n == 0) return;
    with_types(a, [&](auto e, auto te) { launch_forward<decltype(e), decltype(te)>(a, st); });
}

void launch_distil_loss_backward(const DistilArgs &a, hipStream_t st)
{
    if (a.n == 0) return;
    with_types(a, [&](auto e, auto te) { launch_backward<decltype(e), decltype(te)>(a, st); });
}

} // namespace bht
