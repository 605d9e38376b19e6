// Layer norm over the rows (points) of an n x d matrix, forward and backward.
//
//   y = (x - mean) rstd w + b,   rstd = (1/d sum (x - mean)^2 + eps)^(-1/2)
//   g = dy w, xh = (x - mean) rstd:
//   dx = rstd (g - 1/d sum g - xh 1/d sum g xh),  dw = sum_n dy xh,  db = sum_n dy
//
// Both passes move each element once (two or three of them) for about ten
// operations: HBM bounds them.  A row is held in the registers of a team of
// 2^k lanes of a wave (up to 1024 features at 16 a lane), or of a whole block
// (up to 16384; backward, with two rows and the weights' sums, half of both),
// so that the mean, the centred sum of squares and the outputs come from one
// read; the next row's loads are in flight while a row is computed.  A row's sums
// are fp32, of 16 terms a lane at most, and fp64 in longer rows; the weights'
// gradients are summed in fp32 by a block and in fp64 over the blocks.  The only
// rounding to fewer bits is that of the outputs.
#include <type_traits>

#include "map.hpp"

namespace bht {
namespace {

template <typename E, int VEC> struct alignas(sizeof(E) * VEC) Pack {
    E v[VEC];
};

// kStream: 16-byte accesses of rows that do not stay in the caches (kNormStream) leave no lines behind: backward of
// 1.3M x 128 bf16 180 us against 194, forward of 1.3M x 256 257 against 278.  Narrower ones come back to their lines
// and lose by it (70k x 500 by 8 bytes 52 us against 45, both before the parameters came by vectors).
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
template <bool kStream, typename E, int VEC> __device__ inline Pack<E, VEC> load_pack(const E *p)
{
    if constexpr (kStream)
        return __builtin_bit_cast(Pack<E, VEC>, __builtin_nontemporal_load(reinterpret_cast<const uint4v *>(p)));
    else
        return *reinterpret_cast<const Pack<E, VEC> *>(p);
}
template <bool kStream, typename E, int VEC> __device__ inline void store_pack(E *p, const Pack<E, VEC> &v)
{
    if constexpr (kStream)
        __builtin_nontemporal_store(__builtin_bit_cast(uint4v, v), reinterpret_cast<uint4v *>(p));
    else
        *reinterpret_cast<Pack<E, VEC> *>(p) = v;
}

// Weights and their gradients are fp32, or of 16 bits of either kind.  Which is the same for the whole launch, and is
// asked outside of whatever depends on the lane: kWide, in code of its own; the two kinds of 16 bits by a selection.
// (Nested in a lane's condition, such branches have cost an address register its value on one of the paths.)
template <bool kWide> struct Params {
    const void *p;
    bool half; // fp16 rather than bf16
    __device__ float at(int64_t i) const
    {
        using R = typename std::conditional<kWide, float, uint16_t>::type;
        return value(static_cast<const R *>(p)[i], half);
    }
    __device__ static float value(float v, bool) { return v; }
    __device__ static float value(uint16_t raw, bool half)
    {
        const float h = float(__builtin_bit_cast(f16, raw)), b = __uint_as_float(uint32_t(raw) << 16);
        return half ? h : b;
    }
};
template <bool kWide> __device__ inline void store_param(void *p, Elem t, int64_t i, float v)
{
    if constexpr (kWide) {
        static_cast<float *>(p)[i] = v;
    } else {
        const uint16_t h = __builtin_bit_cast(uint16_t, f16(v)), b = __builtin_bit_cast(uint16_t, bf16(v));
        static_cast<uint16_t *>(p)[i] = t == Elem::kF16 ? h : b;
    }
}

// The parameters of a lane's features: kVector, up to 16 bytes at a time, of arrays that are aligned for it and whose
// last vector is full.  Behind the last feature the last one is read, and `fill` taken.
template <bool kWide, bool kVector, int VEC, int NV>
__device__ inline void load_params(const void *p, bool half, int team, int lane, int d, float fill, float (&out)[NV * VEC])
{
    using R = typename std::conditional<kWide, float, uint16_t>::type;
    constexpr int kMost = 16 / int(sizeof(R)), kTake = !kVector ? 1 : VEC < kMost ? VEC : kMost;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < VEC; j += kTake) {
            const int c = (k * team + lane) * VEC + j;
            const auto raw = *reinterpret_cast<const Pack<R, kTake> *>(static_cast<const R *>(p) + (c < d ? c : d - kTake));
#pragma unroll
            for (int i = 0; i < kTake; ++i) {
                const float v = Params<kWide>::value(raw.v[i], half);
                out[k * VEC + j + i] = c < d ? v : fill;
            }
        }
}
// Weight and bias of a lane's features, 1 and 0 without them; both are asked for before either is waited for
template <int VEC, int NV>
__device__ inline void read_params(const void *weight, const void *bias, Elem t, int team, int lane, int d,
                                   float (&w)[NV * VEC], float (&b)[NV * VEC])
{
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) {
        w[i] = 1.0f;
        b[i] = 0.0f;
    }
    if (!weight && !bias) return;
    const void *pw = weight ? weight : bias, *pb = bias ? bias : weight;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(pw) | reinterpret_cast<uintptr_t>(pb);
    const auto both = [&](auto wide, auto vector) {
        load_params<decltype(wide)::value, decltype(vector)::value, VEC, NV>(pw, t == Elem::kF16, team, lane, d, 1.0f, w);
        load_params<decltype(wide)::value, decltype(vector)::value, VEC, NV>(pb, t == Elem::kF16, team, lane, d, 0.0f, b);
    };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    if (t == Elem::kF32) {
        if (VEC > 1 && (bits & (VEC < 4 ? VEC * 4 - 1 : 15)) == 0)
            both(yes, yes);
        else
            both(yes, no);
    } else {
        if (VEC > 1 && (bits & (VEC * 2 - 1)) == 0)
            both(no, yes);
        else
            both(no, no);
    }
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) {
        w[i] = weight ? w[i] : 1.0f;
        b[i] = bias ? b[i] : 0.0f;
    }
}

// v of the lane at the other end of a fixed permutation within 16 lanes
template <int kCtrl> __device__ inline float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xF, 0xF, true));
}

// what a swap of lane groups leaves in its two registers: each group's value in both groups
template <typename V> __device__ inline float both(V r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); }

// Sum over aligned teams of `team` lanes (a power of two up to 64), in every
// lane.  Once all lanes of an aligned half hold that half's sum, any lane of
// the other half will do: mirrors serve for the exchanges over 4 and 8 lanes.
__device__ inline float team_sum(float v, int team)
{
    if (team > 1) v += dpp<0xB1>(v);  // quad_perm 1,0,3,2
    if (team > 2) v += dpp<0x4E>(v);  // quad_perm 2,3,0,1
    if (team > 4) v += dpp<0x141>(v); // row_half_mirror
    if (team > 8) v += dpp<0x140>(v); // row_mirror
    if (team > 16) v = both(__builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    if (team > 32) v = both(__builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return v;
}

// s / count with inv = 1 / count: a product put right by its remainder, as exact as the division and a third of it
__device__ inline float share(float s, float count, float inv)
{
    const float q = s * inv;
    const float r = fmaf(-q, count, s);
    return fabsf(q) < __FLT_MAX__ ? fmaf(r, inv, q) : q; // an infinite quotient has no remainder
}

// x^(-1/2), the approximation put right once
__device__ inline float inverse_root(float x)
{
    const float r = rsqrtf(x);
    const float e = fmaf(-x * r, r, 1.0f);
    return r > 0.0f && r < __FLT_MAX__ ? fmaf(0.5f * r, e, r) : r;
}

// Sum over the team of a row: lanes of a wave (team <= 64), or the whole block.
// `red`: kNormMaxThreads / 64 floats of LDS for this sum alone.
__device__ inline float row_sum(float v, int team, float *red)
{
    v = team_sum(v, team < kWave ? team : kWave);
    if (team <= kWave) return v;
    if (lane_id() == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < team / kWave; ++w) s += red[w];
    return s;
}

// Sum over a block in fp64, for rows whose lanes have many terms: in fp32 a lane's sum of a hundred equal values is off by
// several roundings, all one way (a constant row of 100.3 came out at 0.03 for d = 100000, at 0.24 for 2^20).
// `red`: kNormMaxThreads / 64 doubles of LDS for this sum alone.
__device__ inline double long_sum(double v, double *red)
{
    v = wave_sum(v);
    if (lane_id() == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < int(blockDim.x) / kWave; ++w) s += red[w];
    return s;
}

// The vectors of a lane: the k-th starts at feature (k team + lane) VEC.  All but the last few are full for every
// lane, which is known without looking at the lanes.
template <int VEC> struct Columns {
    int team, lane, d;
    __device__ int at(int k) const { return (k * team + lane) * VEC; }
    __device__ bool has(int k) const { return (k + 1) * team * VEC <= d || at(k) < d; }
};

// ------------------------------------------------------------------ forward
// One read and one write of a row.  70k x 777 fp32 82 us, 5.3 TB/s of HBM; 1.3M x 256 bf16 257 us, 5.2.  Short rows are
// bound by the issue of two row sums each: 1.3M x 50 fp16 69 us, 3.8 TB/s.  One row of 512: 2.4 us, a launch's latency.
template <typename E, int VEC, int NV, bool kStream>
__global__ __launch_bounds__(kNormMaxThreads) void norm_kernel(NormArgs a, int team)
{
    __shared__ float s_red[2][kNormMaxThreads / kWave];
    const int sub = threadIdx.x & (team - 1);      // lane in the team (team is a power of two up to 64) ...
    const int lane = team <= kWave ? sub : threadIdx.x; // ... or in the block
    const int rows = team <= kWave ? int(blockDim.x) / team : 1;
    const int mine = team <= kWave ? int(threadIdx.x) / team : 0;
    const int d = int(a.d);
    const float count = float(d), inv = 1.0f / count, eps = float(a.eps);
    const Columns<VEC> cols = {team, lane, d};

    float w[NV * VEC], b[NV * VEC];
    const int64_t step = int64_t(gridDim.x) * rows;
    int64_t row = int64_t(blockIdx.x) * rows + mine;
    const E *x = static_cast<const E *>(a.x) + row * a.x_stride + lane * VEC;
    E *y = static_cast<E *>(a.out) + row * a.out_stride + lane * VEC;
    Pack<E, VEC> next[NV] = {};
    const auto load = [&]() {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (cols.has(k)) next[k] = load_pack<kStream, E, VEC>(x + k * team * VEC);
    };
    if (row < a.n) load();
    read_params<VEC, NV>(a.weight, a.bias, a.param, team, lane, d, w, b);

    // every lane of a block makes the same number of rounds
    for (int64_t first = int64_t(blockIdx.x) * rows; first < a.n; first += step, row += step) {
        float v[NV * VEC];
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[k * VEC + j] = float(next[k].v[j]); // zero where there are no features
                sum += v[k * VEC + j];
            }
        x += step * a.x_stride;
        if (first + step + rows <= a.n || row + step < a.n) load();
        const float mean = share(row_sum(sum, team, s_red[0]), count, inv);
        float sq = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float part = 0.0f;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[k * VEC + j] -= mean;
                part += v[k * VEC + j] * v[k * VEC + j];
            }
            sq += cols.has(k) ? part : 0.0f;
        }
        const float rstd = inverse_root(share(row_sum(sq, team, s_red[1]), count, inv) + eps);
        if (first + rows <= a.n || row < a.n) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                Pack<E, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) o.v[j] = E(v[k * VEC + j] * rstd * w[k * VEC + j] + b[k * VEC + j]);
                if (cols.has(k)) store_pack<kStream, E, VEC>(y + k * team * VEC, o);
            }
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
        y += step * a.out_stride;
    }
}

// rows longer than a block's registers: one block a row, three passes over it, the last two from the caches at the rate
// of these (2000 x 20000 fp32 117 us, 2.7 TB/s)
template <typename E, int VEC, bool kWide>
__global__ __launch_bounds__(kNormMaxThreads) void norm_long_kernel(NormArgs a)
{
    __shared__ double s_red[2][kNormMaxThreads / kWave];
    const Params<kWide> weight = {a.weight, a.param == Elem::kF16}, bias = {a.bias, a.param == Elem::kF16};
    const int team = blockDim.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E *x = static_cast<const E *>(a.x) + row * a.x_stride;
        E *y = static_cast<E *>(a.out) + row * a.out_stride;
        double sum = 0.0;
        for (int64_t c = int64_t(threadIdx.x) * VEC; c < a.d; c += int64_t(team) * VEC) {
            const Pack<E, VEC> p = load_pack<false, E, VEC>(x + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += double(p.v[j]);
        }
        const double centre = long_sum(sum, s_red[0]) / double(a.d);
        const float mean = float(centre);
        double sq = 0.0;
        for (int64_t c = int64_t(threadIdx.x) * VEC; c < a.d; c += int64_t(team) * VEC) {
            const Pack<E, VEC> p = load_pack<false, E, VEC>(x + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const double c = double(p.v[j]) - centre;
                sq = fma(c, c, sq);
            }
        }
        const float rstd = float(1.0 / sqrt(long_sum(sq, s_red[1]) / double(a.d) + a.eps));
        for (int64_t c = int64_t(threadIdx.x) * VEC; c < a.d; c += int64_t(team) * VEC) {
            const Pack<E, VEC> p = load_pack<false, E, VEC>(x + c);
            Pack<E, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float w = a.weight ? weight.at(c + j) : 1.0f, b = a.bias ? bias.at(c + j) : 0.0f;
                o.v[j] = E((float(p.v[j]) - mean) * rstd * w + b);
            }
            store_pack<false, E, VEC>(y + c, o);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ------------------------------------------------------------------ backward
// the partial row of a block that was alone, which it has written itself, as gradients
template <bool kWide> __device__ inline void finish(const NormArgs &a)
{
    for (int c = threadIdx.x; c < int(a.d); c += blockDim.x) {
        if (a.dweight) store_param<kWide>(a.dweight, a.param, c, a.part[c]);
        if (a.dbias) store_param<kWide>(a.dbias, a.param, c, a.part[a.d + c]);
    }
}

// Each team keeps the sums of its rows' dy xh and dy in registers; a block's
// teams are joined in LDS, in order, into one partial row [2][d] of the block.
// 1.3M x 256 bf16 334 us, 6.0 TB/s of HBM; 70001 x 500 bf16 by 8 bytes 38 us,
// 5.6, part of it from the last cache; 2000 x 128 fp32 4.2 us, latency.
template <typename E, int VEC, int NV, bool kStream>
__global__ __launch_bounds__(kNormMaxThreads) void norm_back_kernel(NormArgs a, int team)
{
    __shared__ float s_red[2][kNormMaxThreads / kWave];
    extern __shared__ float s_part[]; // [rows][team * NV * VEC], where a wave holds several teams or a block several waves
    const int sub = threadIdx.x & (team - 1);
    const int lane = team <= kWave ? sub : threadIdx.x;
    const int rows = team <= kWave ? int(blockDim.x) / team : 1;
    const int mine = team <= kWave ? int(threadIdx.x) / team : 0;
    const int d = int(a.d);
    const float count = float(d), inv = 1.0f / count;
    const Columns<VEC> cols = {team, lane, d};

    float w[NV * VEC], dw[NV * VEC], db[NV * VEC];
    const int64_t step = int64_t(gridDim.x) * rows;
    int64_t row = int64_t(blockIdx.x) * rows + mine;
    const E *x = static_cast<const E *>(a.x) + row * a.x_stride + lane * VEC;
    const E *dy = static_cast<const E *>(a.dy) + row * a.dy_stride + lane * VEC;
    E *dx = static_cast<E *>(a.out) + row * a.out_stride + lane * VEC;
    Pack<E, VEC> nx[NV] = {}, ndy[NV] = {};
    float nmean = 0.0f, nrstd = 0.0f;
    const auto load = [&](int64_t r) {
        nmean = a.mean[r];
        nrstd = a.rstd[r];
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (cols.has(k)) {
                nx[k] = load_pack<kStream, E, VEC>(x + k * team * VEC);
                ndy[k] = load_pack<kStream, E, VEC>(dy + k * team * VEC);
            }
    };
    if (row < a.n) load(row);
    read_params<VEC, NV>(a.weight, nullptr, a.param, team, lane, d, w, db);
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) dw[i] = db[i] = 0.0f;
    for (int64_t first = int64_t(blockIdx.x) * rows; first < a.n; first += step, row += step) {
        const float mean = nmean, rstd = nrstd;
        const bool have = first + rows <= a.n || row < a.n;
        float xh[NV * VEC], g[NV * VEC];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!have || !cols.has(k)) continue;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = k * VEC + j;
                const float t = float(ndy[k].v[j]);
                xh[i] = (float(nx[k].v[j]) - mean) * rstd;
                g[i] = t * w[i];
                dw[i] += t * xh[i];
                db[i] += t;
                s1 += g[i];
                s2 += g[i] * xh[i];
            }
        }
        x += step * a.x_stride;
        dy += step * a.dy_stride;
        if (first + step + rows <= a.n || row + step < a.n) load(row + step);
        s1 = share(row_sum(s1, team, s_red[0]), count, inv);
        s2 = share(row_sum(s2, team, s_red[1]), count, inv);
        if (have && a.out) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (!cols.has(k)) continue;
                Pack<E, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int i = k * VEC + j;
                    o.v[j] = E(rstd * (g[i] - s1 - xh[i] * s2));
                }
                store_pack<kStream, E, VEC>(dx + k * team * VEC, o);
            }
        }
        dx += step * a.out_stride;
    }
    if (!a.part) return;
    const int width = team * NV * VEC;
    for (int which = 0; which < 2; ++which) {
        float *part = a.part + (int64_t(blockIdx.x) * 2 + which) * d;
        if (rows == 1) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (cols.at(k) + j < d) part[cols.at(k) + j] = which ? db[k * VEC + j] : dw[k * VEC + j];
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s_part[mine * width + cols.at(k) + j] = which ? db[k * VEC + j] : dw[k * VEC + j];
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            float s = 0.0f;
            for (int r = 0; r < rows; ++r) s += s_part[r * width + c];
            part[c] = s;
        }
    }
    if (!a.alone) return;
    // the only block: its sums are the gradients
    __syncthreads();
    if (a.param == Elem::kF32)
        finish<true>(a);
    else
        finish<false>(a);
}

// rows longer than a block's registers: dx, one block a row
template <typename E, int VEC, bool kWide>
__global__ __launch_bounds__(kNormMaxThreads) void norm_back_long_kernel(NormArgs a)
{
    __shared__ double s_red[2][kNormMaxThreads / kWave];
    const Params<kWide> weight = {a.weight, a.param == Elem::kF16};
    const int team = blockDim.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E *x = static_cast<const E *>(a.x) + row * a.x_stride;
        const E *dy = static_cast<const E *>(a.dy) + row * a.dy_stride;
        E *dx = static_cast<E *>(a.out) + row * a.out_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        double sum1 = 0.0, sum2 = 0.0;
        for (int64_t c = int64_t(threadIdx.x) * VEC; c < a.d; c += int64_t(team) * VEC) {
            const Pack<E, VEC> p = load_pack<false, E, VEC>(x + c), q = load_pack<false, E, VEC>(dy + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float w = a.weight ? weight.at(c + j) : 1.0f;
                const float g = float(q.v[j]) * w;
                sum1 += double(g);
                sum2 += double(g) * double((float(p.v[j]) - mean) * rstd);
            }
        }
        const float s1 = float(long_sum(sum1, s_red[0]) / double(a.d)), s2 = float(long_sum(sum2, s_red[1]) / double(a.d));
        for (int64_t c = int64_t(threadIdx.x) * VEC; c < a.d; c += int64_t(team) * VEC) {
            const Pack<E, VEC> p = load_pack<false, E, VEC>(x + c), q = load_pack<false, E, VEC>(dy + c);
            Pack<E, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float w = a.weight ? weight.at(c + j) : 1.0f;
                o.v[j] = E(rstd * (float(q.v[j]) * w - s1 - (float(p.v[j]) - mean) * rstd * s2));
            }
            store_pack<false, E, VEC>(dx + c, o);
        }
    }
}

// ... and its weight gradients, before dx is written (dx may be dy): a block
// owns blockDim columns and the rows of its blockIdx.y, whose partial it writes
template <typename E> __global__ __launch_bounds__(256) void norm_back_columns_kernel(NormArgs a)
{
    const int64_t c = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
    if (c >= a.d) return;
    const E *x = static_cast<const E *>(a.x), *dy = static_cast<const E *>(a.dy);
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const float t = float(dy[row * a.dy_stride + c]);
        dw += t * ((float(x[row * a.x_stride + c]) - a.mean[row]) * a.rstd[row]);
        db += t;
    }
    float *part = a.part + int64_t(blockIdx.y) * 2 * a.d;
    part[c] = dw;
    part[a.d + c] = db;
}

// Joins the blocks' partial rows: 32 columns and 32 strands of partial rows a
// block; sums in fp64 and in a fixed order, whatever the blocks' timing.  Bound
// by latency: 250 rows of 2 x 128 4.2 us, 1024 of 2 x 256 5.2.
constexpr int kJoinCols = 32, kJoinStrands = 32;
template <bool kWide>
__global__ __launch_bounds__(kJoinCols *kJoinStrands) void norm_join_kernel(const float *part, int blocks, int64_t d,
                                                                          void *dweight, void *dbias, Elem param)
{
    __shared__ double s_sum[kJoinStrands][kJoinCols + 1];
    const int cx = threadIdx.x % kJoinCols, strand = threadIdx.x / kJoinCols;
    const int64_t c = int64_t(blockIdx.x) * kJoinCols + cx; // column of [dw | db]
    double s = 0.0;
    if (c < 2 * d) {
#pragma unroll 8
        for (int b = strand; b < blocks; b += kJoinStrands) s += double(part[int64_t(b) * 2 * d + c]);
    }
    s_sum[strand][cx] = s;
    __syncthreads();
    s = 0.0;
    for (int k = 0; k < kJoinStrands; ++k) s += s_sum[k][cx];
    if (strand == 0 && c < d && dweight) store_param<kWide>(dweight, param, c, float(s));
    if (strand == 0 && c >= d && c < 2 * d && dbias) store_param<kWide>(dbias, param, c - d, float(s));
}

// ------------------------------------------------------------------ launch shapes
struct Shape {
    int vec, nv, team, block, rows;
    bool in_regs;
    bool alone; // backward: one block
};

// the widest vectors that every row's start and the row length allow, 16 bytes at most
int vector_of(const NormArgs &a)
{
    const int e = elem_bytes(a.type);
    uintptr_t bits = uintptr_t(a.d) * e | reinterpret_cast<uintptr_t>(a.x) | uintptr_t(a.x_stride) * e | 16u;
    if (a.out) bits |= reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.out_stride) * e;
    if (a.dy) bits |= reinterpret_cast<uintptr_t>(a.dy) | uintptr_t(a.dy_stride) * e;
    return int((bits & (~bits + 1)) / e);
}

// How a row is shared out.  A lane does best with some four features and a few vectors (`some`): more rows a wave pass
// through the row sums together, and loads still cover whole lines (1.3M x 50 fp16: 16 lanes of 2 x 2 features 69 us, 32
// of 2 features 101, 64 of 1 187; 2M x 7 fp32: 4 lanes 23 us, 8 lanes 31, 2 lanes 26), backward with 16 bytes (1.3M x 50
// fp16 by eight 101 us, by four 109; 1.3M x 128 fp32 by four 362, by eight 387).  Where rows are too few to fill the
// chip, one vector a lane (2000 x 128 fp32 3.6 us against 3.7).  `most`: features of a lane, 16 forward and 8 backward,
// whose sums take the registers (16 there spill: 300k x 255 fp32 540 us against 190).
Shape shape_of(int vec, int64_t n, int64_t d, int some, int most)
{
    const auto power = [](int64_t x) {
        int p = 1;
        while (p < x) p *= 2;
        return p;
    };
    Shape s;
    s.vec = vec;
    const int64_t vecs = (d + vec - 1) / vec;
    const int few = n <= kNormFewRows || vec > some ? vec : some;
    int64_t team = power((d + few - 1) / few);
    const int64_t least = power(vecs < 4 ? vecs : 4);
    if (team < least) team = least;
    s.team = int(team < kWave ? team : kWave);
    s.nv = 1;
    while (s.nv * vec < most && int64_t(s.team) * s.nv < vecs) s.nv *= 2;
    s.block = 256;
    if (int64_t(s.team) * s.nv < vecs) {
        const int64_t waves = (vecs + int64_t(s.nv) * kWave - 1) / (int64_t(s.nv) * kWave);
        s.team = s.block = int(waves * kWave < kNormMaxThreads ? waves * kWave : kNormMaxThreads);
    }
    s.in_regs = int64_t(s.team) * s.nv >= vecs;
    if (!s.in_regs) s.team = s.block = kNormMaxThreads;
    s.rows = s.team <= kWave ? s.block / s.team : 1;
    s.alone = false;
    return s;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

template <typename E> bool streams(const NormArgs &a) { return a.n * a.d >= kNormStream / int64_t(sizeof(E)); }

// Blocks of the backward pass, a partial row of the weights' gradient each: 1024 threads a CU (70k x 1000 fp16 by blocks
// of 128 94 us, by half as many 103; 3000 x 8000 fp32 by 256 blocks of 1024 56, by 1024 87), and of rows that have a block
// to themselves kNormBackRows at least, so that the partial rows stay
// few beside them (300 x 8000 bf16 21 us, by a block a row 34; by blocks of 12 rows 30).
int64_t back_blocks(int64_t n, int64_t d, const Shape &s)
{
    return s.alone ? 1 : least(ceil_div(n, s.team > kWave ? kNormBackRows : s.rows), norm_back_blocks(n, d));
}

template <typename E, int VEC, int NV> void forward_regs(const NormArgs &a, const Shape &s, hipStream_t st)
{
    const int64_t blocks = least(ceil_div(a.n, s.rows), int64_t(kCus) * (2048 / s.block));
    if constexpr (sizeof(E) * VEC == 16)
        if (streams<E>(a)) {
            norm_kernel<E, VEC, NV, true><<<dim3(uint32_t(blocks)), dim3(s.block), 0, st>>>(a, s.team);
            return;
        }
    norm_kernel<E, VEC, NV, false><<<dim3(uint32_t(blocks)), dim3(s.block), 0, st>>>(a, s.team);
}
template <typename E, int VEC, int NV> void backward_regs(const NormArgs &a, const Shape &s, hipStream_t st)
{
    const int64_t blocks = back_blocks(a.n, a.d, s);
    const size_t lds = s.rows > 1 ? size_t(s.block) * NV * VEC * sizeof(float) : 0;
    if constexpr (sizeof(E) * VEC == 16)
        if (streams<E>(a)) {
            norm_back_kernel<E, VEC, NV, true><<<dim3(uint32_t(blocks)), dim3(s.block), lds, st>>>(a, s.team);
            return;
        }
    norm_back_kernel<E, VEC, NV, false><<<dim3(uint32_t(blocks)), dim3(s.block), lds, st>>>(a, s.team);
}

template <typename E, int VEC> void forward_vec(const NormArgs &a, const Shape &s, hipStream_t st)
{
    if (!s.in_regs) {
        const int64_t blocks = least(a.n, 2 * kCus);
        if (a.param == Elem::kF32)
            norm_long_kernel<E, VEC, true><<<dim3(uint32_t(blocks)), dim3(s.block), 0, st>>>(a);
        else
            norm_long_kernel<E, VEC, false><<<dim3(uint32_t(blocks)), dim3(s.block), 0, st>>>(a);
        return;
    }
    switch (s.nv) {
    case 1: return forward_regs<E, VEC, 1>(a, s, st);
    case 2:
        if constexpr (VEC * 2 <= kNormLane) return forward_regs<E, VEC, 2>(a, s, st);
    case 4:
        if constexpr (VEC * 4 <= kNormLane) return forward_regs<E, VEC, 4>(a, s, st);
    case 8:
        if constexpr (VEC * 8 <= kNormLane) return forward_regs<E, VEC, 8>(a, s, st);
    default:
        if constexpr (VEC * 16 <= kNormLane) return forward_regs<E, VEC, 16>(a, s, st);
    }
}
template <typename E, int VEC> void backward_vec(const NormArgs &a, const Shape &s, hipStream_t st)
{
    if (!s.in_regs) {
        if (a.part) {
            const int64_t blocks = back_blocks(a.n, a.d, s);
            norm_back_columns_kernel<E><<<dim3(uint32_t(ceil_div(a.d, 256)), uint32_t(blocks)), dim3(256), 0, st>>>(a);
        }
        const dim3 grid(uint32_t(least(a.n, 2 * kCus)));
        if (a.out && a.param == Elem::kF32)
            norm_back_long_kernel<E, VEC, true><<<grid, dim3(s.block), 0, st>>>(a);
        else if (a.out)
            norm_back_long_kernel<E, VEC, false><<<grid, dim3(s.block), 0, st>>>(a);
        return;
    }
    switch (s.nv) {
    case 1: return backward_regs<E, VEC, 1>(a, s, st);
    case 2:
        if constexpr (VEC * 2 <= kNormLaneBack) return backward_regs<E, VEC, 2>(a, s, st);
    case 4:
        if constexpr (VEC * 4 <= kNormLaneBack) return backward_regs<E, VEC, 4>(a, s, st);
    default:
        if constexpr (VEC * 8 <= kNormLaneBack) return backward_regs<E, VEC, 8>(a, s, st);
    }
}

Shape shape_of(const NormArgs &a, bool back)
{
    // Few rows are shared out over more lanes forward too (8000 x 1000 fp32 11.4 us against 13.2), which no longer pays
    // for long ones (8000 x 3333 bf16 34.1 us against 30.4)
    const bool narrow = back || (a.n <= kNormFewRows && a.d <= kNormFewFeatures);
    Shape s = shape_of(vector_of(a), a.n, a.d, back ? 16 / elem_bytes(a.type) : 4, narrow ? kNormLaneBack : kNormLane);
    // Few rows backward: one large block goes over them in less than the launch takes that joins several (250 x 128
    // fp32 12.4 us a call against 14.8; a row of several waves takes 2 us a round, 8 x 4000 bf16 17.5 against 14.7)
    const int rows = s.team <= kWave ? kNormMaxThreads / s.team : 1;
    if (back && s.in_regs && a.n > 0 && a.n <= int64_t(s.team <= kWave ? kNormAlone : kNormAlone / 2) * rows) {
        s.alone = true;
        s.rows = rows;
        if (s.team <= kWave) s.block = kNormMaxThreads;
    }
    return s;
}

template <bool kBack, typename E> void run_type(const NormArgs &a, hipStream_t st)
{
    const Shape s = shape_of(a, kBack);
    const auto go = [&](auto vec) {
        if constexpr (kBack)
            backward_vec<E, decltype(vec)::value>(a, s, st);
        else
            forward_vec<E, decltype(vec)::value>(a, s, st);
    };
    if constexpr (sizeof(E) == 2)
        if (s.vec == 8) return go(std::integral_constant<int, 8>());
    if (s.vec == 4) return go(std::integral_constant<int, 4>());
    if (s.vec == 2) return go(std::integral_constant<int, 2>());
    return go(std::integral_constant<int, 1>());
}

template <bool kBack> void run_norm(const NormArgs &a, hipStream_t st)
{
    if (a.type == Elem::kF32)
        run_type<kBack, float>(a, st);
    else if (a.type == Elem::kF16)
        run_type<kBack, f16>(a, st);
    else
        run_type<kBack, bf16>(a, st);
}

} // namespace

void launch_layer_norm(const NormArgs &a, hipStream_t st)
{
    if (a.n > 0) run_norm<false>(a, st);
}

void launch_layer_norm_backward(const NormArgs &args, hipStream_t st)
{
    NormArgs a = args;
    const Shape s = shape_of(a, true);
    a.alone = s.alone;
    if (a.n > 0) run_norm<true>(a, st);
    if (!a.part || a.alone) return;
    const int blocks = int(back_blocks(a.n, a.d, s));
    const dim3 grid(uint32_t(ceil_div(2 * a.d, kJoinCols)));
    if (a.param == Elem::kF32)
        norm_join_kernel<true><<<grid, kJoinCols * kJoinStrands, 0, st>>>(a.part, blocks, a.d, a.dweight, a.dbias, a.param);
    else
        norm_join_kernel<false><<<grid, kJoinCols * kJoinStrands, 0, st>>>(a.part, blocks, a.d, a.dweight, a.dbias, a.param);
}

} // namespace bht
