// A gated hidden layer: h = act(a) b with a = x gate^T, b = x up^T, and its backward pass.
//
// Forward is one product of x with both matrices: a wave holds a and b of the same
// points and features in its registers, so the activation and the product are its
// epilogue, and neither a nor b has to go to memory (they are written, rounded once,
// where the backward pass will take them).  Bound by the matrix cores: 16384 x 2048 to
// 8192 bf16 with a and b, 1.1 TFLOP and 805 MB written, 836 us (1.32 PFLOP/s); they are
// busy 73 % of it, and rest while a tile's outputs are formed, some 6 of 52 us.
//
// Backward, with a and b as they were kept:
//   da = dh b act'(a), db = dh act(a);  dx = da gate + db up;  dgate = da^T x, dup = db^T x
// da and db are formed once, in fp32, and rounded to the inputs' type, as operands of
// matrix instructions of that type: with bf16 their rounding adds to the output's own
// (1.7e-3 each, 2.4e-3 together).  Where outputs are few and the products small, that
// average does not hold for them and operands of 32 bits cost little: they are fp32
// (kFewOutputs).  The sums over features and points are fp32.
#include <cmath>

#include "products.hpp"

namespace bht {
namespace {

using namespace prod;

// ------------------------------------------------------------------ activations
// fp32 with the library's exponential; 16-bit outputs do not show the instruction's last bits
template <typename E> __device__ inline float sigmoid(float a)
{
    if constexpr (sizeof(E) == 4)
        return 1.0f / (1.0f + expf(-a));
    else
        return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a * -1.44269504f));
}
// Half of erfc(|a| / sqrt(2)) = exp(-a^2 / 2) t P(t) with t = 1 / (1 + c |a|): P is fitted to the scaled function over all
// |a| by least squares, reweighted towards the largest relative error: of degree 8 for fp32 (1.3e-7; with its own roundings
// 4.6e-7), of degree 5 for outputs of 16 bits (1.8e-5, a twenty-seventh of fp16's rounding).  No difference of near values, so
// a far below zero keeps its digits.  The exponential is a square, so that values near the smallest fp32 and bf16 numbers do
// not vanish in the instruction.
template <typename E> __device__ inline float tail(float a, float &root)
{
    constexpr bool kWide = sizeof(E) == 4;
    constexpr int kDegree = kWide ? 8 : 5;
    constexpr float kWideP[9] = {0.11283793300390244f, 0.11283478140830994f, 0.10392161458730698f, 0.08426911383867264f, 0.07072257250547409f,
                                 -0.0028178293723613024f, 0.08455897867679596f, -0.09146063029766083f, 0.0251335259526968f};
    constexpr float kNarrowP[9] = {0.12976588308811188f, 0.12951643764972687f, 0.12026726454496384f, 0.06271062791347504f, 0.12091848254203796f, -0.06318359076976776f};
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(a), kWide ? 0.28284273f : 0.32526913f, 1.0f));
    float p = kWide ? kWideP[8] : kNarrowP[5];
#pragma unroll
    for (int k = kDegree - 1; k >= 0; --k) p = fmaf(p, t, kWide ? kWideP[k] : kNarrowP[k]);
    root = __builtin_amdgcn_exp2f(a * (a * -0.360673760f));
    return p * t * root * root;
}
// (value) a Phi(a) and (slope) Phi(a) + a phi(a); or the sigmoid's.  Phi is the tail or one less it, and a its factor: max(a, 0) -
// |a| tail(a) is an instruction less (1.3M x 50 to 200 fp16 263 us for 270), but infinity less infinity times 0 above zero.
__device__ inline float phi_of(float a, float h) { return a < 0.0f ? h : 1.0f - h; }
template <typename E> __device__ inline float activate(float a, Act act)
{
    if (act == Act::kSilu) return a * sigmoid<E>(a);
    float root;
    return a * phi_of(a, tail<E>(a, root));
}
template <typename E> __device__ inline void activate_both(float a, Act act, float &value, float &slope)
{
    if (act == Act::kSilu) {
        const float s = sigmoid<E>(a);
        value = a * s;
        slope = s * (1.0f + a * (1.0f - s));
    } else {
        float root;
        const float phi = phi_of(a, tail<E>(a, root));
        value = a * phi;
        slope = phi + a * (0.398942280f * root * root);
    }
}

// ------------------------------------------------------------------ forward
struct GatedOut {
    void *h, *a, *b;
    int64_t h_stride, a_stride, b_stride;
    Act act;
    bool vec_h, vec_a, vec_b, inner;
};

// A tile inside the outputs
template <typename E, typename T, Act kAct, bool kKeep>
__device__ inline void put_inner(int32_t bi, int32_t bj, const GatedOut &o, const typename Ops<E>::Acc (&acc)[T::kI][T::kJ])
{
    typedef InnerRuns<T, Form::kDual> Runs;
    constexpr int kRun = Runs::kTogether;
    const Runs runs(bi, bj);
    const auto to_h = runs.template to<E>(o.h, o.h_stride), to_a = runs.template to<E>(o.a, o.a_stride), to_b = runs.template to<E>(o.b, o.b_stride);
#pragma unroll
    for (int i = 0; i < T::kI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float a[kRun], b[kRun], h[kRun];
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                a[e] = acc[i][e][r];
                b[e] = acc[i][kRun + e][r];
                h[e] = activate<E>(a[e], kAct) * b[e];
            }
            to_h.put(i, r, h);
            if constexpr (kKeep) {
                to_a.put(i, r, a);
                to_b.put(i, r, b);
            }
        }
}

template <typename E, typename T, bool kAny, Tail kTail>
__global__ __launch_bounds__(T::kThreads) void gated_kernel(Product p, GatedOut o)
{
    constexpr int kRun = T::kJ / 2; // features of a lane
    each_tile<E, T, Form::kDual, kAny, kTail>(p, [&](int32_t bi, int32_t bj, typename Ops<E>::Acc (&acc)[T::kI][T::kJ]) {
        if (o.inner && tile_inside<T, Form::kDual>(p, bi, bj)) {
            if (o.act == Act::kSilu)
                return o.a ? put_inner<E, T, Act::kSilu, true>(bi, bj, o, acc) : put_inner<E, T, Act::kSilu, false>(bi, bj, o, acc);
            return o.a ? put_inner<E, T, Act::kGelu, true>(bi, bj, o, acc) : put_inner<E, T, Act::kGelu, false>(bi, bj, o, acc);
        }
        each_run<T, Form::kDual>(bi, bj, [&](int64_t point, int64_t feature, int i, int r) {
            if (point >= p.rows) return;
            float a[kRun], b[kRun], h[kRun];
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                a[e] = acc[i][e][r];
                b[e] = acc[i][kRun + e][r];
                h[e] = activate<E>(a[e], o.act) * b[e];
            }
            const int64_t count = p.features - feature;
            store_run(static_cast<E *>(o.h) + point * o.h_stride + feature, h, count, o.vec_h);
            if (o.a) store_run(static_cast<E *>(o.a) + point * o.a_stride + feature, a, count, o.vec_a);
            if (o.b) store_run(static_cast<E *>(o.b) + point * o.b_stride + feature, b, count, o.vec_b);
        });
    });
}

template <typename E, int kRun> GatedOut gated_out(const GatedArgs &a)
{
    GatedOut o = {};
    o.h = a.h;
    o.a = a.a;
    o.b = a.b;
    o.h_stride = a.h_stride;
    o.a_stride = a.a_stride;
    o.b_stride = a.b_stride;
    o.act = a.act;
    o.vec_h = runs_aligned<E, kRun>(a.h, a.h_stride);
    o.vec_a = runs_aligned<E, kRun>(a.a, a.a_stride);
    o.vec_b = runs_aligned<E, kRun>(a.b, a.b_stride);
    o.inner = runs_inner<E, kRun>(a.h, a.h_stride) && runs_inner<E, kRun>(a.a, a.a_stride) && runs_inner<E, kRun>(a.b, a.b_stride)
              && (a.a == nullptr) == (a.b == nullptr);
    return o;
}

Product gated_product(const GatedArgs &a, int64_t es)
{
    Product p = {};
    p.A = static_cast<const char *>(a.x);
    p.B = static_cast<const char *>(a.gate);
    p.B2 = static_cast<const char *>(a.up);
    p.a_stride = a.x_stride * es;
    p.b_stride = a.gate_stride * es;
    p.b2_stride = a.up_stride * es;
    p.rows = a.n;
    p.features = a.f;
    p.bytes = a.d * es;
    p.slices = p.per_split = int32_t((p.bytes + kSlice - 1) / kSlice);
    return p;
}

template <typename E, typename T, bool kAny, Tail kTail = Tail::kWhole> void run_gated(const GatedArgs &a, hipStream_t st)
{
    constexpr int64_t kF = T::kN / 2;
    Product p = gated_product(a, int64_t(sizeof(E)));
    p.across = int32_t((a.f + kF - 1) / kF);
    const size_t lds = size_t(kAny && p.slices == 1 ? 1 : T::kStages) * T::kBuffer;
    const int64_t most = kMostTiles / p.across > 0 ? kMostTiles / p.across * T::kM : T::kM; // points of a launch
    for (int64_t from = 0; from < a.n; from += most) {
        p.A = static_cast<const char *>(a.x) + from * p.a_stride;
        p.rows = a.n - from < most ? a.n - from : most;
        p.down = int32_t((p.rows + T::kM - 1) / T::kM);
        GatedOut o = gated_out<E, T::kJ / 2>(a);
        o.h = static_cast<E *>(a.h) + from * a.h_stride;
        o.a = a.a ? static_cast<E *>(a.a) + from * a.a_stride : nullptr;
        o.b = a.b ? static_cast<E *>(a.b) + from * a.b_stride : nullptr;
        gated_kernel<E, T, kAny, kTail><<<blocks_of<T>(uint32_t(p.down) * uint32_t(p.across)), T::kThreads, lds, st>>>(p, o);
    }
}

// Short rows (16 to kHalves 64 bytes): a block holds the weights of up to kShortFeatures features in LDS, and each wave
// takes 16 points at a time past all of them, with no barrier: the points' pieces in registers, the next ones under way, the
// weights' read for each 32 features, whose outputs go through a patch of LDS of the wave's own and from there as 16 bytes a
// lane, runs of 64 bytes of a point.  A row's last piece is its last 16 bytes, of which only those count that the piece before
// does not have: the others are masked out, in points and weights alike.
//
// 1.3M x 50 to 200 fp16, gelu: 245 to 270 us for 650 MB, by the card.  Bound by the vector instructions, which a CU issues in
// 92 % of the time: some 18 an output for the activation and the product, two of them at a quarter of the rate, and 7 blocks
// of 32 features for 6.25.  Rows of 400 bytes end inside a line, so 608 MB are written for 520.  Weights in registers and the
// points past a block's waves in step, by LDS and a barrier, took 301 us (7 waves on 4 SIMDs); without LDS, 429: each lane's
// 16 bytes a request of its own.
constexpr int kShortFeatures = 256; // of a block at most
constexpr int kShortThreads = 512;
constexpr int kShortBlocks = 2 * 2 * kCus;
constexpr int kShortPitch(int kHalves) { return kHalves * 64 + 16; } // bytes of a row of weights in LDS: 8 rows on different banks

struct ShortShape {
    int64_t per_wave; // points, a multiple of 16
    int32_t features; // of a block, a multiple of 32
};

// What lanes of a wave have put into LDS is there for its other lanes.  A wave's LDS accesses keep their order, so this
// costs no instruction: it holds the compiler to that order.
__device__ inline void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename E, int kHalves, bool kGelu, bool kKeep>
__global__ __launch_bounds__(kShortThreads) void gated_short_kernel(Product p, GatedOut o, ShortShape z)
{
    extern __shared__ __align__(16) char s_mem[];
    constexpr int kPitch = kShortPitch(kHalves), kRowPieces = kHalves * 4, kOuts = kKeep ? 3 : 1, kV = 16 / int(sizeof(E));
    constexpr int kPatch = 32 * int(sizeof(E)) + 16; // bytes of a point's 32 outputs in LDS
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();
    const int64_t block = int64_t(blockIdx.y) * z.features;
    const int features = int(p.features - block < z.features ? p.features - block : z.features);
    const int bytes = int(p.bytes);
    char *patch = s_mem + 2 * z.features * kPitch + w * (16 * kPatch);
    // the place of piece c of a row, and what of it counts
    const auto place_of = [&](int c, Piece &mask) {
        const int begin = c * 16, at = begin < bytes - 16 ? begin : bytes - 16, skip = begin - at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int part = skip - 4 * e;
            mask[e] = part <= 0 ? -1 : part >= 4 ? 0 : int(0xffffffffu << (8 * part));
        }
        return at;
    };
    // Weights: 32 features are four blocks of 16 rows, gate's even and odd features, then up's
    for (int e = int(threadIdx.x); e < 2 * z.features * kRowPieces; e += kShortThreads) {
        const int row = e / kRowPieces, c = e % kRowPieces, j = row / 16 % 4;
        const int64_t f = block + row / 64 * 32 + row % 16 * 2 + j % 2, held = f < p.features ? f : p.features - 1;
        Piece mask;
        const int at = place_of(c, mask);
        *reinterpret_cast<Piece *>(s_mem + row * kPitch + c * 16) = inner_piece((j < 2 ? p.B + held * p.b_stride : p.B2 + held * p.b2_stride) + at) & mask;
    }
    __syncthreads();
    const int64_t from = (int64_t(blockIdx.x) * (kShortThreads / kWave) + w) * z.per_wave, to = from + z.per_wave < p.rows ? from + z.per_wave : p.rows;
    if (from >= to) return;
    Piece mask[kHalves], x[kHalves], y[kHalves];
    int at[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) at[h] = place_of(h * 4 + lane / 16, mask[h]);
    const auto load = [&](const char *row, Piece (&v)[kHalves]) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) v[h] = inner_piece(row + at[h]);
    };
    int64_t point = from + lane % 16; // that is loaded
    const char *row = p.A + (point < p.rows ? point : p.rows - 1) * p.a_stride;
    load(row, y);
    // outputs: this lane's 16 bytes of the patch, and where they go
    constexpr int kEach = 32 / kV; // vectors of a point
    const int out_row = lane / kEach, out_column = lane % kEach * kV; // rows of a store: 64 / kEach
    const bool vec = o.vec_h && (!kKeep || (o.vec_a && o.vec_b));
    for (int64_t first = from; first < to; first += 16, point += 16) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) x[h] = y[h] & mask[h];
        if (first + 32 <= p.rows)
            row += 16 * p.a_stride;
        else
            row = p.A + (point + 16 < p.rows ? point + 16 : p.rows - 1) * p.a_stride;
        load(row, y);
        const int rows = int(to - first < 16 ? to - first : 16);
        const char *in = s_mem + lane % 16 * kPitch + lane / 16 * 16;
        for (int f = 0; f < features; f += 32, in += 64 * kPitch) {
            typename Ops<E>::Acc acc[4] = {};
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = Ops<E>::mul(x[h], *reinterpret_cast<const Piece *>(in + j * 16 * kPitch + h * 64), acc[j]);
#pragma unroll
            for (int k = 0; k < kOuts; ++k) {
                typedef typename std::conditional<sizeof(E) == 2, uint32_t, uint64_t>::type Bits;
                struct Two {
                    E v[2];
                };
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    Two t;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float a = acc[e][r], b = acc[2 + e][r];
                        t.v[e] = rounded<E>(k == 0 ? activate<E>(a, kGelu ? Act::kGelu : Act::kSilu) * b : k == 1 ? a : b);
                    }
                    *reinterpret_cast<Bits *>(patch + (lane / 16 * 4 + r) * kPatch + lane % 16 * 2 * int(sizeof(E))) = __builtin_bit_cast(Bits, t);
                }
                wave_exchange();
                E *out = static_cast<E *>(k == 0 ? o.h : k == 1 ? o.a : o.b);
                const int64_t stride = k == 0 ? o.h_stride : k == 1 ? o.a_stride : o.b_stride;
                out += first * stride + block + f;
                if (vec) {
#pragma unroll
                    for (int q = 0; q < 16 * kEach / kWave; ++q) {
                        const int r = out_row + q * (kWave / kEach);
                        const Piece v = *reinterpret_cast<const Piece *>(patch + r * kPatch + out_column * int(sizeof(E)));
                        E *to_out = out + r * stride + out_column;
                        if (f + 32 <= features) {
                            if (r < rows) *reinterpret_cast<Piece *>(to_out) = v;
                        } else if (r < rows) {
                            const int count = features - f - out_column;
                            if (count >= kV) {
                                *reinterpret_cast<Piece *>(to_out) = v;
                            } else {
#pragma unroll
                                for (int e = 0; e < kV; ++e)
                                    if (e < count) to_out[e] = *reinterpret_cast<const E *>(patch + r * kPatch + (out_column + e) * int(sizeof(E)));
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const int r = q * 2 + lane / 32, c = lane % 32;
                        const E v = *reinterpret_cast<const E *>(patch + r * kPatch + c * int(sizeof(E)));
                        if (r < rows && f + c < features) out[r * stride + c] = v;
                    }
                }
                wave_exchange(); // the patch is written again
            }
        }
    }
}

int64_t tiles_of(int64_t rows, int64_t cols, int m, int n) { return (rows + m - 1) / m * ((cols + n - 1) / n); }

// A few points (few_points): 1 x 512 to 2048 bf16 4.4 us, of which a launch is 2.5.
template <typename E, int kI> __global__ __launch_bounds__(kFewWaves *kWave) void gated_few_kernel(Product p, GatedOut o)
{
    __shared__ float s_sum[kFewWaves][2][kI][256];
    const int64_t feature = int64_t(blockIdx.x) * 16, first = int64_t(blockIdx.y) * (16 * kI);
    const int lane = lane_id();
    const char *row[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const int64_t point = first + 16 * i + lane % 16;
        row[i] = p.A + (point < p.rows ? point : p.rows - 1) * p.a_stride;
    }
    const auto x = [&](int32_t slice, int half, int i) {
        const int64_t k = int64_t(slice) * kSlice + half * 64 + lane / 16 * 16;
        return int64_t(slice + 1) * kSlice <= p.bytes ? inner_piece(row[i] + k) : any_piece<E>(row[i], k, p.bytes);
    };
    typename Ops<E>::Acc acc[2][kI] = {};
    few_points<E, 2, kI>(p, feature, [] {}, x, acc);
    few_put(acc, s_sum);
    for (int t = int(threadIdx.x); t < 256 * kI; t += kFewWaves * kWave) {
        const int64_t point = first + t / 16, at = feature + t % 16;
        if (point >= p.rows || at >= p.features) continue;
        const float a = few_sum(s_sum, 0, t / 256, t % 256), b = few_sum(s_sum, 1, t / 256, t % 256);
        static_cast<E *>(o.h)[point * o.h_stride + at] = rounded<E>(activate<E>(a, o.act) * b);
        if (o.a) static_cast<E *>(o.a)[point * o.a_stride + at] = E(a);
        if (o.b) static_cast<E *>(o.b)[point * o.b_stride + at] = E(b);
    }
}
template <typename E, int kI> void run_gated_few(const GatedArgs &a, hipStream_t st)
{
    const dim3 grid(uint32_t((a.f + 15) / 16), uint32_t((a.n + 16 * kI - 1) / (16 * kI)));
    gated_few_kernel<E, kI><<<grid, kFewWaves * kWave, 0, st>>>(gated_product(a, int64_t(sizeof(E))), gated_out<E, 1>(a));
}

template <typename E, int kHalves> void run_gated_short(const GatedArgs &a, hipStream_t st)
{
    constexpr int kEs = int(sizeof(E)), kWaves = kShortThreads / kWave;
    const Product p = gated_product(a, kEs);
    const GatedOut o = gated_out<E, 16 / kEs>(a);
    const bool keep = a.a != nullptr;
    const int64_t groups = (a.f + kShortFeatures - 1) / kShortFeatures;
    ShortShape z = {};
    z.features = int32_t(((a.f + groups - 1) / groups + 31) / 32 * 32);
    const int64_t across = (a.f + z.features - 1) / z.features;
    // a few rounds of two blocks a CU
    const int64_t want = (kShortBlocks + across - 1) / across * kWaves, most = (a.n + want - 1) / want;
    z.per_wave = (most + 15) / 16 * 16;
    const int64_t waves = (a.n + z.per_wave - 1) / z.per_wave;
    const dim3 grid(uint32_t((waves + kWaves - 1) / kWaves), uint32_t(across));
    const size_t lds = 2 * size_t(z.features) * kShortPitch(kHalves) + size_t(kWaves) * 16 * (32 * kEs + 16);
    const auto launch = [&](auto kernel) { kernel<<<grid, kShortThreads, lds, st>>>(p, o, z); };
    if (a.act == Act::kGelu)
        keep ? launch(gated_short_kernel<E, kHalves, true, true>) : launch(gated_short_kernel<E, kHalves, true, false>);
    else
        keep ? launch(gated_short_kernel<E, kHalves, false, true>) : launch(gated_short_kernel<E, kHalves, false, false>);
}

template <typename E> void run_gated_type(const GatedArgs &a, hipStream_t st)
{
    const int64_t es = int64_t(sizeof(E));
    if (a.n <= kFewPoints) return run_gated_few<E, 1>(a, st);
    if (a.d * es >= 16 && a.d * es <= 128 && (a.a == nullptr) == (a.b == nullptr))
        return a.d * es <= 64 ? run_gated_short<E, 1>(a, st) : run_gated_short<E, 2>(a, st);
    const bool any = !aligned16(a.x, a.x_stride * es) || !aligned16(a.gate, a.gate_stride * es) || !aligned16(a.up, a.up_stride * es)
                     || a.d * es % 16 != 0;
    if (few_tiles(a.n, a.f, !any || es == 4)) return run_gated_few<E, kFewRows / 16>(a, st);
    const bool near = a.x_stride * es <= kLargeStride && a.gate_stride * es <= kLargeStride && a.up_stride * es <= kLargeStride;
    const Side side = plan_product(a.n, 2 * a.f, slices_of(a.d * es), es == 4, false, any || !near ? Side::kMiddle : Side::kLarge).side;
    if (any) {
        if (side == Side::kMiddle) return run_gated<E, TileMiddle, true>(a, st);
        return run_gated<E, TileSmall, true>(a, st);
    }
    if (side == Side::kLarge) return a.d * es % kSlice == 0 ? run_gated<E, TileLarge, false, Tail::kWhole>(a, st) : run_gated<E, TileLarge, false, Tail::kZeros>(a, st);
    if (side == Side::kMiddle) return run_gated<E, TileMiddle, false>(a, st);
    run_gated<E, TileSmall, false>(a, st);
}

// ------------------------------------------------------------------ backward: operands
// One launch: da and db side by side, a row a point; the weights transposed and side by side; x with rows that are padded to
// 16 bytes, where its own are not.  Blocks are dealt to the three by their number.  Bound by HBM: 70000 x 512 to 2048 bf16,
// 0.86 GB read and 0.58 written, 276 us.
constexpr int kT = 64; // side of a tile that is transposed

struct Operands {
    const void *dh, *a, *b, *x, *gate, *up;
    char *d, *xp, *wt;
    int64_t dh_stride, a_stride, b_stride, x_stride, gate_stride, up_stride;
    int64_t n, features, f;
    int64_t np, fp, dp, ld;         // padded; from row to row of d
    uint32_t slope_blocks, weight_blocks, x_blocks;
    Act act;
    bool straight;                  // rows of f values of dh, a and b are whole pieces
};

template <typename E> __device__ inline Piece row_piece(const void *p, int64_t row_bytes, int64_t row, int64_t c, int64_t bytes, bool straight)
{
    const char *r = static_cast<const char *>(p) + row * row_bytes;
    return straight ? inner_piece(r + c * 16) : any_piece<E>(r, c * 16, bytes);
}

// C: of the operands, E or fp32
template <typename E, typename C> __global__ __launch_bounds__(256) void gated_operands_kernel(Operands g)
{
    constexpr int kEs = int(sizeof(E)), kCs = int(sizeof(C)), kV = 16 / kEs; // values at a time
    struct alignas(16) Values {
        E v[kV];
    };
    struct alignas(16) Made {
        C v[kV];
    };
    __shared__ C s_t[kT][kT + 2];
    uint32_t b = blockIdx.x;
    if (b >= g.weight_blocks && b < g.weight_blocks + g.slope_blocks) {
        b -= g.weight_blocks;
        const int64_t each = g.fp / kV, total = g.np * each;
        for (int64_t t = int64_t(b) * 256 + threadIdx.x; t < total; t += int64_t(g.slope_blocks) * 256) {
            const int64_t row = total <= 0xffffffffll ? uint32_t(t) / uint32_t(each) : t / each, c = t - row * each;
            const int64_t bytes = g.f * kEs;
            char *out = g.d + (row * g.ld + c * kV) * kCs;
            if (row >= g.n || c * kV >= g.f) { // padding
                *reinterpret_cast<Made *>(out) = Made{};
                *reinterpret_cast<Made *>(out + g.fp * kCs) = Made{};
                continue;
            }
            const Values dh = __builtin_bit_cast(Values, row_piece<E>(g.dh, g.dh_stride * kEs, row, c, bytes, g.straight));
            const Values av = __builtin_bit_cast(Values, row_piece<E>(g.a, g.a_stride * kEs, row, c, bytes, g.straight));
            const Values bv = __builtin_bit_cast(Values, row_piece<E>(g.b, g.b_stride * kEs, row, c, bytes, g.straight));
            Made da, db;
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                float value, slope;
                activate_both<E>(float(av.v[e]), g.act, value, slope);
                const float d = float(dh.v[e]);
                da.v[e] = C(d * float(bv.v[e]) * slope);
                db.v[e] = C(d * value);
            }
            *reinterpret_cast<Made *>(out) = da;
            *reinterpret_cast<Made *>(out + g.fp * kCs) = db;
        }
        return;
    }
    if (b < g.weight_blocks) {
        const uint32_t across = uint32_t((g.features + kT - 1) / kT), down = uint32_t((g.fp + kT - 1) / kT);
        const bool second = b >= across * down;
        if (second) b -= across * down;
        const E *in = static_cast<const E *>(second ? g.up : g.gate);
        const int64_t stride = second ? g.up_stride : g.gate_stride, r0 = int64_t(b / across) * kT, c0 = int64_t(b % across) * kT;
        constexpr int kEach = kT * kT / 256;
        const int col = int(threadIdx.x) % kT, row = int(threadIdx.x) / kT; // every fourth row; all loads asked for at once
        E v[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int64_t r = r0 + row + q * (256 / kT), c = c0 + col;
            v[q] = in[(r < g.f ? r : g.f - 1) * stride + (c < g.features ? c : g.features - 1)];
        }
#pragma unroll
        for (int q = 0; q < kEach; ++q) s_t[row + q * (256 / kT)][col] = r0 + row + q * (256 / kT) < g.f ? C(float(v[q])) : C(0.0f);
        __syncthreads();
        C *out = reinterpret_cast<C *>(g.wt) + (second ? g.fp : 0);
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int c = row + q * (256 / kT);
            if (r0 + col < g.fp && c0 + c < g.features) out[(c0 + c) * 2 * g.fp + r0 + col] = s_t[col][c];
        }
        return;
    }
    b -= g.weight_blocks + g.slope_blocks;
    const int64_t each = g.dp / kV, total = g.n * each;
    for (int64_t t = int64_t(b) * 256 + threadIdx.x; t < total; t += int64_t(g.x_blocks) * 256) {
        const int64_t row = total <= 0xffffffffll ? uint32_t(t) / uint32_t(each) : t / each, c = t - row * each;
        const Values x = __builtin_bit_cast(Values, any_piece<E>(static_cast<const char *>(g.x) + row * g.x_stride * kEs, c * 16, g.features * kEs));
        Made y;
#pragma unroll
        for (int e = 0; e < kV; ++e) y.v[e] = C(float(x.v[e]));
        *reinterpret_cast<Made *>(g.xp + t * (kV * kCs)) = y;
    }
}

// ------------------------------------------------------------------ backward: products
// dx: rows as they are.  The weights' gradients: rows 0 .. f - 1 are dgate's, rows from `first2` on dup's (dx: none are).
// kPart: fp32 partial sums of a split, of 2 f rows (dx: of n).  70000 x 512 to 2048 bf16, 0.29 TFLOP each: dx 284 us, whose
// 550 tiles are three rounds of CUs, the weights 262 to 318 (1.1 to 0.9 PFLOP/s) by the card, and 14 to join 8 parts; their
// operands' rows are read across (kColumns), which costs no copy of da, db and x on its other side (with one 1417 us a pass,
// so 991 then).
struct BackOut {
    void *out, *out2;
    float *part;
    int64_t stride, stride2, first2, f, features; // f: rows of an output
    int64_t part_rows;
    bool vec, inner;
};

// C: of the operands, E: of the outputs
template <typename E, typename C, typename T, Form kForm, bool kPart>
__global__ __launch_bounds__(T::kThreads) void gated_back_kernel(Product p, BackOut o)
{
    constexpr int kRun = T::kJ;
    each_tile<C, T, kForm, false, Tail::kWhole>(p, [&](int32_t bi, int32_t bj, typename Ops<C>::Acc (&acc)[T::kI][T::kJ]) {
        if constexpr (kForm == Form::kRows) {
            if (o.inner && tile_inside<T, kForm>(p, bi, bj)) {
                typedef std::conditional_t<kPart, float, E> Out;
                const auto to = InnerRuns<T, kForm>(bi, bj).template to<Out>(kPart ? o.part + int64_t(blockIdx.y) * o.part_rows * o.features : o.out,
                                                                             kPart ? o.features : o.stride);
#pragma unroll
                for (int i = 0; i < T::kI; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v[kRun];
#pragma unroll
                        for (int e = 0; e < kRun; ++e) v[e] = acc[i][e][r];
                        to.put(i, r, v);
                    }
                return;
            }
        }
        each_run<T, kForm>(bi, bj, [&](int64_t row, int64_t feature, int i, int r) {
            if (row >= p.rows) return;
            float v[kRun];
#pragma unroll
            for (int e = 0; e < kRun; ++e) v[e] = acc[i][e][r];
            const int64_t count = o.features - feature; // p.features may be padded
            if constexpr (kForm == Form::kRows) {
                if constexpr (kPart)
                    store_run(o.part + (int64_t(blockIdx.y) * o.part_rows + row) * o.features + feature, v, count, o.vec);
                else
                    store_run(static_cast<E *>(o.out) + row * o.stride + feature, v, count, o.vec);
            } else {
                const bool second = row >= o.first2;
                const int64_t at = second ? row - o.first2 : row;
                E *out = static_cast<E *>(second ? o.out2 : o.out);
                if (at >= o.f) return;
#pragma unroll
                for (int e = 0; e < kRun; ++e) {
                    if (16 * e >= count) continue;
                    if constexpr (kPart)
                        o.part[(int64_t(blockIdx.y) * o.part_rows + (second ? o.f : 0) + at) * o.features + feature + 16 * e] = v[e];
                    else if (out)
                        out[at * (second ? o.stride2 : o.stride) + feature + 16 * e] = E(v[e]);
                }
            }
        });
    });
}

// The splits' sums in a fixed order, fp64: two values a thread where rows have an even number
template <typename E, int kV> __global__ __launch_bounds__(256) void gated_join_kernel(BackOut o, int splits)
{
    struct alignas(4 * kV) Part {
        float v[kV];
    };
    struct alignas(sizeof(E) * kV) Out {
        E v[kV];
    };
    const int64_t each = o.features / kV, total = o.part_rows * each;
    const Part *part = reinterpret_cast<const Part *>(o.part);
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < total; e += int64_t(gridDim.x) * 256) {
        double sum[kV] = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const Part x = part[s * total + e];
#pragma unroll
            for (int k = 0; k < kV; ++k) sum[k] += double(x.v[k]);
        }
        const int64_t row = total <= 0xffffffffll ? uint32_t(e) / uint32_t(each) : e / each, col = (e - row * each) * kV;
        const bool second = row >= o.f;
        E *out = static_cast<E *>(second ? o.out2 : o.out);
        if (!out) continue;
        out += (second ? row - o.f : row) * (second ? o.stride2 : o.stride) + col;
        Out y;
#pragma unroll
        for (int k = 0; k < kV; ++k) y.v[k] = E(float(sum[k]));
        *reinterpret_cast<Out *>(out) = y;
    }
}

template <typename E, typename C, typename T, Form kForm>
void run_back(Product p, const BackOut &o, int splits, hipStream_t st)
{
    p.slices = int32_t(slices_of(p.bytes));
    p.per_split = (p.slices + splits - 1) / splits;
    p.across = int32_t((p.features + T::kN - 1) / T::kN);
    const size_t lds = size_t(T::kStages) * T::kBuffer;
    const int64_t all = p.rows, most = kMostTiles / p.across > 0 ? kMostTiles / p.across * T::kM : T::kM;
    const char *A = p.A;
    for (int64_t from = 0; from < all; from += most) { // several launches only of kRows without splits: others have fewer tiles
        p.A = A + from * p.a_stride;
        p.rows = all - from < most ? all - from : most;
        p.down = int32_t((p.rows + T::kM - 1) / T::kM);
        BackOut q = o;
        if (kForm == Form::kRows) q.out = static_cast<E *>(o.out) + from * o.stride;
        const dim3 grid(blocks_of<T>(uint32_t(p.down) * uint32_t(p.across)), uint32_t(splits));
        if (splits > 1)
            gated_back_kernel<E, C, T, kForm, true><<<grid, T::kThreads, lds, st>>>(p, q);
        else
            gated_back_kernel<E, C, T, kForm, false><<<grid, T::kThreads, lds, st>>>(p, q);
    }
}

template <typename E, typename C, Form kForm> void run_back_plan(const Product &p, BackOut o, Plan plan, hipStream_t st)
{
    constexpr int64_t es = int64_t(sizeof(E));
    o.part_rows = kForm == Form::kRows ? o.f : 2 * o.f;
    const bool pairs = o.features % 2 == 0 && aligned_to(2 * es, o.out, o.stride * es) && aligned_to(2 * es, o.out2, o.stride2 * es);
    if (plan.splits > 1) o.vec = o.features % 4 == 0; // of the partial sums
    o.inner = o.vec && (plan.splits > 1 ? o.features * 4 : o.stride * es) <= kLargeStride;
    if constexpr (!std::is_same<E, C>::value)
        run_back<E, C, TileSmall, kForm>(p, o, plan.splits, st);
    else if (plan.side == Side::kLarge)
        run_back<E, C, TileLarge, kForm>(p, o, plan.splits, st);
    else if (plan.side == Side::kMiddle)
        run_back<E, C, TileMiddle, kForm>(p, o, plan.splits, st);
    else
        run_back<E, C, TileSmall, kForm>(p, o, plan.splits, st);
    if (plan.splits == 1) return;
    const int64_t blocks = (o.part_rows * o.features / (pairs ? 2 : 1) + 255) / 256;
    const uint32_t grid = uint32_t(blocks < 16384 ? blocks : 16384);
    if (pairs)
        gated_join_kernel<E, 2><<<grid, 256, 0, st>>>(o, plan.splits);
    else
        gated_join_kernel<E, 1><<<grid, 256, 0, st>>>(o, plan.splits);
}

template <typename E, typename C> void run_gated_back_of(const GatedBackArgs &a, const GatedBackLayout &L, hipStream_t st)
{
    const int64_t es = int64_t(sizeof(E)), cs = int64_t(sizeof(C)), kV = 16 / es;
    char *ws = static_cast<char *>(a.ws);
    const bool weights = a.dgate || a.dup, pad_x = weights && (cs != es || !aligned16(a.x, a.x_stride * es) || a.d * es % 16 != 0 || a.x_stride * es > kLargeStride);
    Operands g = {};
    g.dh = a.dh;
    g.a = a.a;
    g.b = a.b;
    g.x = a.x;
    g.gate = a.gate;
    g.up = a.up;
    g.dh_stride = a.dh_stride;
    g.a_stride = a.a_stride;
    g.b_stride = a.b_stride;
    g.x_stride = a.x_stride;
    g.gate_stride = a.gate_stride;
    g.up_stride = a.up_stride;
    g.n = a.n;
    g.features = a.d;
    g.f = a.f;
    g.np = L.np;
    g.ld = L.ld;
    g.fp = L.fp;
    g.dp = L.dp;
    g.d = ws + L.d;
    g.xp = ws + L.xp;
    g.wt = ws + L.wt;
    g.act = a.act;
    g.straight = a.f * es % 16 == 0;
    const auto blocks_for = [](int64_t pieces) {
        const int64_t blocks = (pieces + 255) / 256;
        return uint32_t(blocks < 16 * kCus ? blocks : 16 * kCus);
    };
    g.slope_blocks = blocks_for(L.np * (L.fp / kV));
    g.weight_blocks = a.dx ? uint32_t(2 * tiles_of(L.fp, a.d, kT, kT)) : 0;
    g.x_blocks = pad_x ? blocks_for(a.n * (L.dp / kV)) : 0;
    gated_operands_kernel<E, C><<<g.slope_blocks + g.weight_blocks + g.x_blocks, 256, 0, st>>>(g);
    if (a.dx) {
        Product p = {};
        p.A = g.d;
        p.B = g.wt;
        p.a_stride = L.ld * cs;
        p.b_stride = p.bytes = 2 * L.fp * cs;
        p.rows = a.n;
        p.features = a.d;
        BackOut o = {};
        o.out = a.dx;
        o.stride = a.dx_stride;
        o.first2 = int64_t(1) << 62;
        o.f = a.n;
        o.features = a.d;
        o.part = reinterpret_cast<float *>(ws + L.part);
        o.vec = aligned16(a.dx, a.dx_stride * es);
        run_back_plan<E, C, Form::kRows>(p, o, L.x, st);
    }
    if (weights) {
        Product p = {};
        p.A = g.d;
        p.B = pad_x ? g.xp : static_cast<const char *>(a.x);
        p.a_stride = L.ld * cs;
        p.b_stride = (pad_x ? L.dp : a.x_stride) * cs;
        p.bytes = a.n * cs;
        p.rows = 2 * L.fp;
        p.features = pad_x ? L.dp : a.d;
        BackOut o = {};
        o.out = a.dgate;
        o.out2 = a.dup;
        o.stride = a.dgate_stride;
        o.stride2 = a.dup_stride;
        o.first2 = L.fp;
        o.f = a.f;
        o.features = a.d;
        o.part = reinterpret_cast<float *>(ws + L.part);
        run_back_plan<E, C, Form::kColumns>(p, o, L.weights, st);
    }
}

template <typename E> void run_gated_back(const GatedBackArgs &a, hipStream_t st)
{
    const GatedBackLayout L = make_gated_back_layout(a.n, a.d, a.f, a.type);
    L.wide ? run_gated_back_of<E, float>(a, L, st) : run_gated_back_of<E, E>(a, L, st);
}

template <typename E> __global__ __launch_bounds__(256) void gated_zero_kernel(E *p, int64_t stride, int64_t rows, int64_t cols)
{
    const int64_t total = rows * cols;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < total; e += int64_t(gridDim.x) * 256)
        p[e / cols * stride + e % cols] = E(0.0f);
}

// no points: the weights' gradients are zero
template <typename E> void run_gated_zero(const GatedBackArgs &a, hipStream_t st)
{
    const int64_t blocks = (a.f * a.d + 255) / 256;
    const uint32_t grid = uint32_t(blocks < 8192 ? blocks : 8192);
    if (a.dgate) gated_zero_kernel<E><<<grid, 256, 0, st>>>(static_cast<E *>(a.dgate), a.dgate_stride, a.f, a.d);
    if (a.dup) gated_zero_kernel<E><<<grid, 256, 0, st>>>(static_cast<E *>(a.dup), a.dup_stride, a.f, a.d);
}

} // namespace

// By the time of the busiest CU, in us, from what slices took of 8-bit products (fp32's matrix instructions take eight times as
// long, which is all that counts there).  A tile of 256 alone on a CU: 1.0, and 1.42 with all CUs at it.  One of 128: 0.73,
// two on a CU 1.1, and so on by half that each.  One of 64: 0.32, two 0.45, then 0.2 each.  A tile's start and end take 9, 5 and
// 2.5; joining partial sums a launch and their bytes.
Plan plan_product(int64_t rows, int64_t columns, int64_t slices, bool wide, bool may_split, Side most)
{
    const auto slice_time = [&](Side side, int64_t blocks) {
        const int64_t each = (blocks + kCus - 1) / kCus; // of the busiest CU
        if (wide) return double(each) * (side == Side::kSmall ? 0.46 : side == Side::kMiddle ? 1.75 : 6.9);
        if (side == Side::kLarge) return each > 1 ? 1.42 * double(each) : 1.0 + 0.42 * double(blocks) / kCus;
        if (side == Side::kMiddle) return each > 1 ? 0.55 * double(each) : 0.73;
        return each > 2 ? 0.2 * double(each) + 0.05 : each > 1 ? 0.45 : 0.32;
    };
    Plan best = {Side::kSmall, 1};
    double least = INFINITY;
    for (const Side side : {Side::kSmall, Side::kMiddle, Side::kLarge}) {
        if (int(side) > int(most)) continue;
        const int64_t tiles = tiles_of(rows, columns, int(side), int(side));
        const double fixed = side == Side::kSmall ? 2.5 : side == Side::kMiddle ? 5.0 : 9.0;
        const int at_once = side == Side::kSmall ? 3 * kCus : side == Side::kMiddle ? 2 * kCus : kCus;
        for (int want = 1; want <= (may_split ? kMostSplits : 1); want += want < 8 ? 1 : want / 4) {
            const int64_t per = (slices + want - 1) / want;
            if (per < 1 || (want > 1 && per < 4)) break;
            const int splits = int((slices + per - 1) / per);
            if (side == Side::kLarge && (per < 2 || slices - (splits - 1) * per < 2)) continue;
            if (splits > 1 && splits * rows * columns * 4 > kMostPart) break;
            const int64_t blocks = tiles * splits, rounds = (blocks + at_once - 1) / at_once;
            const double t = fixed * double(rounds) + double(per) * slice_time(side, blocks)
                             + (splits > 1 ? 4.0 + double(splits) * double(rows) * double(columns) * 8.0 / 4.5e6 : 0.0);
            if (t < least) {
                least = t;
                best = {side, splits};
            }
        }
    }
    return best;
}

// The rounding of 16-bit operands is as large as that of the outputs, 1.41 times it together where sums are of many unlike
// terms; over a few outputs that can come out at twice it (bf16, dx of 100 values 3.0e-3 against 1.6e-3).  So small products of
// few outputs take fp32 operands (2^27 points x features x features are 7 us of matrix instructions).
constexpr int64_t kFewOutputs = 4096;
constexpr double kFewProducts = 134217728.0;

GatedBackLayout make_gated_back_layout(int64_t n, int64_t d, int64_t f, Elem type)
{
    GatedBackLayout L = {};
    L.wide = type == Elem::kF32 || ((n * d < kFewOutputs || f * d < kFewOutputs) && double(n) * double(d) * double(f) < kFewProducts);
    const int es = L.wide ? 4 : 2;
    L.fp = (f * es + kSlice - 1) / kSlice * kSlice / es;
    L.np = (n * es + kSlice - 1) / kSlice * kSlice / es;
    L.dp = pad16(d, elem_bytes(type)); // of the inputs' pieces
    const Side most = L.wide && type != Elem::kF32 ? Side::kSmall : Side::kLarge; // small products gain nothing by more
    L.x = plan_product(n, d, slices_of(2 * L.fp * es), es == 4, true, most);
    L.weights = plan_product(2 * L.fp, d, slices_of(n * es), es == 4, true, most);
    size_t at = 0;
    const auto take = [&](int64_t count, int bytes) {
        const size_t here = at;
        at += (size_t(count) * size_t(bytes) + 255) / 256 * 256;
        return here;
    };
    L.ld = 2 * L.fp + 256 / es; // rows side by side in other channels of the caches
    L.d = take(L.np * L.ld, es);
    L.xp = take(n * L.dp, es);
    L.wt = take(d * 2 * L.fp, es);
    const int64_t x_part = L.x.splits > 1 ? L.x.splits * n * d : 0, w_part = L.weights.splits > 1 ? L.weights.splits * 2 * f * d : 0;
    L.part = take(x_part > w_part ? x_part : w_part, 4);
    L.total = at > 0 ? at : 256;
    return L;
}

void launch_gated_layer(const GatedArgs &a, hipStream_t st)
{
    if (a.n == 0) return;
    if (a.type == Elem::kF32) return run_gated_type<float>(a, st);
    if (a.type == Elem::kF16) return run_gated_type<f16>(a, st);
    run_gated_type<bf16>(a, st);
}

void launch_gated_layer_backward(const GatedBackArgs &a, hipStream_t st)
{
    if (a.type == Elem::kF32) return a.n == 0 ? run_gated_zero<float>(a, st) : run_gated_back<float>(a, st);
    if (a.type == Elem::kF16) return a.n == 0 ? run_gated_zero<f16>(a, st) : run_gated_back<f16>(a, st);
    a.n == 0 ? run_gated_zero<bf16>(a, st) : run_gated_back<bf16>(a, st);
}

} // namespace bht
