// Orthogonalisation of a matrix by Newton-Schulz products, and the momentum step
// of a weight matrix with it.
//
//   M <- mu M + G,  U = G + mu M (Nesterov) or M      (or U = G alone)
//   X = U / (|U|_F + eps), shorter side first (m <= n)
//   k times:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//   W <- keep W - rate X                              (or the output is X)
//
// The products run on the matrix cores with fp16 operands and fp32 sums.  X is
// held as two fp16 halves (22 bits together) times a power of two that keeps
// every value of the step inside fp16's range.  Small singular values grow by a
// factor of a each step against the largest, and the largest come out of terms
// that cancel, so each product is three, high by high and the two mixed ones, for
// outputs of every type.  a X is added to B X in fp32: as part of B, a I would
// round with B's small values beside it, and matrices of low rank or of values that
// fall off would lose by it (against 64 bits, eight directions over noise, 1024 x
// 1030: 5.3e-5, apart 3.0e-5; the formula in 32 bits, term by term, 4.5e-5).  So
// the result is as far from 64 bits as the formula in 32 bits, 1.2 times at most in
// what was measured: 1e-6 to 2e-6 for gaussian values, 2e-4 for rank 1.
#include <type_traits>

#include "map.hpp"

namespace bht {
namespace {

typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kT = 64; // tile of the planes' kernel

// ------------------------------------------------------------------ norm and planes
__device__ inline float update_value(const OrthArgs &a, float g, float m)
{
    return a.M ? (a.nesterov != 0.0f ? g + a.momentum * m : m) : g;
}

// Eight values of a row from p, of which `left` exist; vec: p and the row are aligned for 16-byte loads
template <typename E> struct alignas(16) Vec16 {
    E v[16 / sizeof(E)];
};
template <typename E> __device__ inline void load8(const E *p, int left, bool vec, float (&v)[8])
{
    constexpr int kV = 16 / sizeof(E);
    if (vec && left >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / kV; ++h) {
            const Vec16<E> x = reinterpret_cast<const Vec16<E> *>(p)[h];
#pragma unroll
            for (int e = 0; e < kV; ++e) v[h * kV + e] = float(x.v[e]);
        }
        return;
    }
    // the last value again behind the end, and nothing of a row that does not exist
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (left <= 0) return;
    E x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[e < left ? e : left - 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? float(x[e]) : 0.0f;
}
__device__ inline void store8(float *p, int left, bool vec, const float (&v)[8])
{
    if (vec && left >= 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) p[e] = v[e];
}

// The momentum's update, and partial sums of U's squares: fp64, in a fixed order.  One read of G (and M, written back):
// 4096 x 4096 bf16 16 us, 2.1 TB/s, 16 rounds of a thread with one load in flight each; 1024 x 1024 3.5 us, a launch's latency.
template <typename E>
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs a, char *ws, int64_t ws_stride, size_t at)
{
    __shared__ double s_w[256 / kWave];
    const int64_t z = blockIdx.y;
    double sum = 0.0;
    const uint32_t across = uint32_t((a.cols + 7) / 8), total = across * uint32_t(a.rows); // < 2^29
    for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < total; e += gridDim.x * 256) {
        const uint32_t r = e / across, c = (e - r * across) * 8;
        const int left = a.cols - c < 8 ? int(a.cols - c) : 8;
        float g[8], m[8] = {};
        load8(static_cast<const E *>(a.G) + z * a.g_batch + r * a.g_stride + c, left, a.g_vec, g);
        if (a.M) {
            float *M = a.M + z * a.m_batch + r * a.m_stride + c;
            load8(M, left, a.m_vec, m);
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = a.momentum * m[k] + g[k];
            store8(M, left, a.m_vec, m);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const double u = double(update_value(a, g[k], m[k]));
            sum += u * u;
        }
    }
    sum = wave_sum(sum);
    if (lane_id() == 0) s_w[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < 256 / kWave; ++w) t += s_w[w];
        reinterpret_cast<double *>(ws + z * ws_stride + at)[blockIdx.x] = t;
    }
}

__device__ inline void split(float v, f16 &h, f16 &l)
{
    h = f16(v);
    l = f16(v - float(h));
}

// U / (|U| + eps) in planes, in both orientations, zeros in the padding.  Where |U| is far below eps, X is small and
// stays small, and fp16 would lose it: it is held larger by a power of two, 1 / `lift`, such that no step passes its
// bound.  Only A and the output are formed with `lift`; the products that lead from X to X are linear in it.
// Bound by HBM: 4096 x 4096 bf16 34 us for 134 MB written and 34 read (4.9 TB/s); 1024 x 1024 11 us, of which the partial
// norms and the first values are some 3 of latency.
template <typename E>
__global__ __launch_bounds__(256) void orth_planes_kernel(OrthArgs a, char *ws, OrthLayout L, int norm_blocks, float sx, double reach)
{
    __shared__ float s_t[kT][kT + 1];
    const int64_t z = blockIdx.z, r0 = int64_t(blockIdx.y) * kT, c0 = int64_t(blockIdx.x) * kT;
    char *base = ws + z * L.stride;
    const int piece = threadIdx.x % 8 * 8;
    float v[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int64_t r = r0 + threadIdx.x / 8 + 32 * s, c = c0 + piece;
        const int left = r < a.rows ? int(a.cols - c) : 0;
        float m[8] = {};
        load8(static_cast<const E *>(a.G) + z * a.g_batch + r * a.g_stride + c, left, a.g_vec, v[s]);
        if (a.M) load8(a.M + z * a.m_batch + r * a.m_stride + c, left, a.m_vec, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[s][e] = update_value(a, v[s][e], m[e]);
    }
    const double *part = reinterpret_cast<const double *>(base + L.norm);
    double sq = 0.0;
#pragma unroll
    for (int q = 0; q < kOrthNormBlocks / kWave; ++q) { // all asked for at once
        const int k = q * kWave + lane_id();
        const double v = part[k < norm_blocks ? k : 0];
        sq += k < norm_blocks ? v : 0.0;
    }
    sq = wave_sum(sq);
    const double norm = sqrt(sq), inverse = 1.0 / (norm + a.eps);
    double scale = double(sx) * inverse;
    const double top = norm * inverse * reach; // what |X| can reach beside its bounds, which allow 1
    if (top > 0.0 && top < 0.5) {
        constexpr int kMostLift = 110; // its inverse is a normal float, with digits to spare for the output
        const int e = -ilogb(top) - 1;
        const double up = ldexp(1.0, e < kMostLift ? e : kMostLift);
        scale *= up;
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *reinterpret_cast<float *>(base + L.lift) = float(1.0 / up);
    } else if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        *reinterpret_cast<float *>(base + L.lift) = 1.0f;
    }
    f16 *uh = reinterpret_cast<f16 *>(base + L.u[0]), *ul = uh + L.rows * L.cols;
    f16 *vh = reinterpret_cast<f16 *>(base + L.v[0]), *vl = vh + L.rows * L.cols;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int row = threadIdx.x / 8 + 32 * s;
        const int64_t at = (r0 + row) * L.cols + c0 + piece;
        half8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = float(double(v[s][e]) * scale);
            f16 xh, xl;
            split(x, xh, xl);
            h[e] = xh;
            l[e] = xl;
            s_t[row][piece + e] = x;
        }
        *reinterpret_cast<half8 *>(uh + at) = h;
        *reinterpret_cast<half8 *>(ul + at) = l;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int col = threadIdx.x / 8 + 32 * s;
        half8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f16 xh, xl;
            split(s_t[piece + e][col], xh, xl);
            h[e] = xh;
            l[e] = xl;
        }
        *reinterpret_cast<half8 *>(vh + (c0 + col) * L.rows + r0 + piece) = h;
        *reinterpret_cast<half8 *>(vl + (c0 + col) * L.rows + r0 + piece) = l;
    }
}

// ------------------------------------------------------------------ products
enum class Prod { kGram, kPoly, kApply, kLast };

// A block makes a kM x kN tile of C = P Q^T, P and Q row-major with K values a row, by kWm x kWn waves.  Slices of
// 64 values a row (128 bytes) go through a ring of kStages buffers in LDS, filled by loads that write LDS directly,
// kStages slices ahead.  A row's eight 16-byte pieces are stored in an order that depends on the row (piece c of
// row r in place c ^ (r % 8)), so that the lanes of a fragment read, which take the same piece of 16 rows, fall on
// different banks.  Tiles may hang over the padded sides: their loads repeat the last row, nothing is stored there.
//
// 4096 x 4096: symmetric products 315 us by tiles of 64 (0.65 PFLOP/s of the half that is computed, the other half is
// stored from it; matrix cores busy 40 % of the time), X' 400 us by tiles of 128 (1.0 PFLOP/s, 48 %): bound by the loop,
// in which every wave of a CU reads and multiplies at the same time (below).  1024 x 1024: 14.0 and 13.6 us, of which a
// launch is 2.5 and the first slices 1.3.
constexpr int kK = 64;
typedef float float4v __attribute__((ext_vector_type(4)));
template <int M, int N, int Wm, int Wn, int Stages> struct Tile {
    static constexpr int kM = M, kN = N, kWm = Wm, kWn = Wn, kStages = Stages;
    static constexpr int kWaves = Wm * Wn, kThreads = kWaves * kWave;
    static constexpr int kI = M / Wm / 16, kJ = N / Wn / 16;   // 16 x 16 blocks of a wave
    static constexpr int kGroups = (M + N) / 8;                // groups of 8 rows in a stage and plane, P's first
    static constexpr int kEach = kGroups / kWaves;             // groups a wave loads
    static constexpr int kHigh = kI % 3 == 0 ? 3 : kI % 2 == 0 ? 2 : 1; // blocks down a patch of the output
    static constexpr int kPatch = 16 * kJ + 1;                 // its row in LDS, floats
    static_assert(kGroups % kWaves == 0 && M % (16 * Wm) == 0 && N % (16 * Wn) == 0, "even shares");
};

// What lanes of a wave have put into LDS is there for its other lanes.  A wave's LDS accesses keep their order, so this
// costs no instruction: it holds the compiler to that order.
__device__ inline void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ inline half8 fragment(const f16 *tile, int row, int piece)
{
    return *reinterpret_cast<const half8 *>(tile + row * kK + ((piece ^ (row & 7)) * 8));
}

// Logical tile of a block: blocks are dealt to the 8 XCDs in turn, each XCD gets consecutive tiles
__device__ inline int xcd_tile(int b, int blocks)
{
    const int x = b % 8, q = blocks / 8, r = blocks % 8;
    return x * q + (x < r ? x : r) + b / 8;
}

// What a product's blocks take.  The first 64 bytes are what the loop waits for: one line of the arguments, with the
// pointers and quotients made on the host, so that the first loads are on their way early (with one product of halves
// for three, 1024 x 1024 took 127 us a pass against 131, 512 x 512 71 against 75).
struct alignas(64) OrthProduct {
    const f16 *P, *Q;         // of the first matrix
    int64_t stride;           // bytes between matrices
    int64_t p_plane, q_plane; // values between high and low halves
    int32_t K, p_rows, q_rows; // padded
    int32_t tiles, across;    // of a matrix, and of four rows of tiles (not of symmetric products)
    uint32_t per_four;        // 2^32 / across rounded up: t across < 2^32 for every tile t
    f16 *out, *out_t;         // C and its transpose in planes
    const f16 *old;           // A of kPoly, X of kApply and kLast
    const float *lift;        // kGram and kLast: of the first matrix
    int64_t out_plane;
    int32_t ld, ld_t;
    float f_c, f_old;         // C becomes f_c C + f_old old
    // kLast: the weights, or the output
    float keep, rate;
    int32_t update, rows, cols;
    void *W;
    int64_t w_batch, w_stride;
};

// E: elements of the output of kLast
template <typename T, Prod kProd, typename E>
__global__ __launch_bounds__(T::kThreads) void orth_product_kernel(OrthProduct a)
{
    constexpr int kPlanes = 2;
    constexpr int kPlane = (T::kM + T::kN) * kK;           // values of a staged plane: P's rows, then Q's
    constexpr int kLoads = kPlanes * T::kEach;             // of a wave and stage
    constexpr bool kSymmetric = kProd == Prod::kGram || kProd == Prod::kPoly;
    extern __shared__ __align__(16) char s_mem[];
    f16 *ring = reinterpret_cast<f16 *>(s_mem);
    const int64_t shift = int64_t(blockIdx.z) * (a.stride / int64_t(sizeof(f16)));
    const f16 *P = a.P + shift, *Q = a.Q + shift;
    float lift = 1.0f;
    if constexpr (kProd == Prod::kGram || kProd == Prod::kLast)
        lift = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(a.lift) + int64_t(blockIdx.z) * a.stride);
    const int K = a.K, p_rows = a.p_rows, q_rows = a.q_rows;
    int bi, bj;
    const int t = xcd_tile(blockIdx.x, a.tiles);
    if constexpr (kSymmetric) {
        // tiles on and below the diagonal, row by row
        bi = int((__builtin_amdgcn_sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
        while (bi * (bi + 1) / 2 > t) --bi;
        bj = t - bi * (bi + 1) / 2;
    } else {
        // four rows of tiles at a time, column by column
        const int down = (p_rows + T::kM - 1) / T::kM;
        const int group = int(__umulhi(uint32_t(t), a.per_four)), top = group * 4;
        const int in = t - group * a.across;
        if (down - top >= 4) {
            bi = top + in % 4;
            bj = in / 4;
        } else {
            const int high = down - top;
            bi = top + in % high;
            bj = in / high;
        }
    }
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();

    // this lane's piece of each group of eight rows that the wave loads
    const f16 *src[kLoads];
#pragma unroll
    for (int e = 0; e < T::kEach; ++e) {
        const int row = (e * T::kWaves + w) * 8 + lane / 8;
        const bool in_p = (e * T::kWaves + w) * 8 < T::kM;
        int at = in_p ? bi * T::kM + row : bj * T::kN + row - T::kM;
        const int most = (in_p ? p_rows : q_rows) - 1;
        at = at < most ? at : most;
        src[e] = (in_p ? P : Q) + int64_t(at) * K + ((lane % 8) ^ (lane / 8)) * 8;
        src[T::kEach + e] = src[e] + (in_p ? a.p_plane : a.q_plane);
    }
    const int slices = K / kK;
    const auto fetch = [&](int slice) {
        // past the end the last slice again, into a buffer that nobody reads: every wait counts alike
        const int64_t k0 = int64_t(slice < slices ? slice : slices - 1) * kK;
        f16 *to = ring + slice % T::kStages * (kPlanes * kPlane);
#pragma unroll
        for (int h = 0; h < kPlanes; ++h)
#pragma unroll
            for (int e = 0; e < T::kEach; ++e)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)(src[h * T::kEach + e] + k0),
                    (__attribute__((address_space(3))) void *)(to + h * kPlane + (e * T::kWaves + w) * 8 * kK), 16, 0, 0);
    };
    const int wi = w / T::kWn * (T::kI * 16), wj = w % T::kWn * (T::kJ * 16);
    // Two sets of fragments.  The second half of a slice is multiplied while the next slice's first is read.  The first
    // half's products wait for both halves: the waits in the assembly below are not the compiler's, which still counts
    // the first half's reads as under way and has one wait for all.  In the middle of a slice both of its halves have
    // been read, by every wave after the barrier, so its buffer is filled again there, and the next slice, which has
    // landed, is read from there on.
    float4v acc[T::kI][T::kJ] = {};
    half8 p[2][kPlanes][T::kI], q[2][kPlanes][T::kJ];
    const auto read = [&](int slice, int half) {
        const f16 *in = ring + slice % T::kStages * (kPlanes * kPlane);
        const int piece = half * 4 + lane / 16;
#pragma unroll
        for (int h = 0; h < kPlanes; ++h) {
#pragma unroll
            for (int i = 0; i < T::kI; ++i) p[half][h][i] = fragment(in + h * kPlane, wi + 16 * i + lane % 16, piece);
#pragma unroll
            for (int j = 0; j < T::kJ; ++j)
                q[half][h][j] = fragment(in + h * kPlane + T::kM * kK, wj + 16 * j + lane % 16, piece);
        }
    };
    const auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i)
#pragma unroll
            for (int j = 0; j < T::kJ; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[half][0][i], q[half][0][j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[half][0][i], q[half][1][j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[half][1][i], q[half][0][j], acc[i][j], 0, 0, 0);
            }
    };
#pragma unroll
    for (int e = 0; e < T::kStages; ++e) fetch(e);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((T::kStages - 1) * kLoads) : "memory");
    read(0, 0);
    for (int slice = 0; slice < slices; ++slice) {
        read(slice, 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);
        // this wave's loads of the next slice have landed and its reads of this one are done; then everybody's
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((T::kStages - 2) * kLoads) : "memory");
        fetch(slice + T::kStages);
        read(slice + 1, 0); // behind the last slice: a buffer of repeated loads, not used
        __builtin_amdgcn_sched_barrier(0);
        multiply(1);
        __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); // the ring is free

    // Each wave puts its blocks through a patch of its own in LDS, for rows of 16 bytes in either orientation
    constexpr int kDown = 16 * T::kHigh, kAcross = 16 * T::kJ;
    float *patch = reinterpret_cast<float *>(s_mem) + w * kDown * T::kPatch;
    f16 *out = a.out + shift, *out_t = a.out_t + shift;
    const f16 *old = a.old + shift;
    const int64_t ld = a.ld, ld_t = a.ld_t, out_plane = a.out_plane;
    const float f_c = kProd == Prod::kGram ? a.f_c * (lift * lift) : a.f_c, f_old = a.f_old; // too small an A is zero
#pragma unroll
    for (int i0 = 0; i0 < T::kI; i0 += T::kHigh) {
        const int r0 = bi * T::kM + wi + 16 * i0, c0 = bj * T::kN + wj;
#pragma unroll
        for (int i = 0; i < T::kHigh; ++i)
#pragma unroll
            for (int j = 0; j < T::kJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    patch[(16 * i + 4 * (lane / 16) + r) * T::kPatch + 16 * j + lane % 16] = acc[i0 + i][j][r];
        wave_exchange();
        if constexpr (kProd == Prod::kLast) {
#pragma unroll 4
            for (int s = 0; s < kDown * T::kJ / 4; ++s) {
                // 16 values of four rows
                const int row = s / T::kJ * 4 + lane / 16, col = s % T::kJ * 16 + lane % 16;
                const int64_t r = r0 + row, c = c0 + col;
                if (r >= a.rows || c >= a.cols) continue;
                const float x = float(old[r * ld + c]) + float(old[out_plane + r * ld + c]);
                const float v = (patch[row * T::kPatch + col] * f_c + f_old * x) * lift;
                E *o = static_cast<E *>(a.W) + int64_t(blockIdx.z) * a.w_batch + r * a.w_stride + c;
                *o = E(a.update ? a.keep * float(*o) - a.rate * v : v);
            }
            wave_exchange(); // the patch is written again
            continue;
        }
        constexpr int kPieces = kDown * kAcross / 8;
#pragma unroll
        for (int s = 0; s < (kPieces + kWave - 1) / kWave; ++s) {
            const int e = lane + kWave * s, row = e / (kAcross / 8), col = e % (kAcross / 8) * 8;
            if (e >= kPieces || r0 + row >= p_rows || c0 + col >= q_rows) continue;
            const int64_t at = (r0 + row) * ld + c0 + col;
            float *v = patch + row * T::kPatch + col;
            half8 h, l, xh, xl;
            if constexpr (kProd != Prod::kGram) {
                xh = *reinterpret_cast<const half8 *>(old + at);
                xl = *reinterpret_cast<const half8 *>(old + out_plane + at);
            }
#pragma unroll
            for (int x8 = 0; x8 < 8; ++x8) {
                float x = v[x8];
                x *= f_c;
                if constexpr (kProd != Prod::kGram) x += f_old * (float(xh[x8]) + float(xl[x8]));
                f16 vh, vl;
                split(x, vh, vl);
                h[x8] = vh;
                l[x8] = vl;
                v[x8] = x;
            }
            *reinterpret_cast<half8 *>(out + at) = h;
            *reinterpret_cast<half8 *>(out + out_plane + at) = l;
        }
        wave_exchange(); // the values of C are there, in either orientation; without one the patch is written again
        if (kSymmetric && bi == bj) continue;
#pragma unroll
        for (int s = 0; s < (kPieces + kWave - 1) / kWave; ++s) {
            const int e = lane + kWave * s, col = e / (kDown / 8), row = e % (kDown / 8) * 8;
            if (e >= kPieces || r0 + row >= p_rows || c0 + col >= q_rows) continue;
            const int64_t at = (c0 + col) * ld_t + r0 + row;
            half8 h, l;
#pragma unroll
            for (int x8 = 0; x8 < 8; ++x8) {
                f16 vh, vl;
                split(patch[(row + x8) * T::kPatch + col], vh, vl);
                h[x8] = vh;
                l[x8] = vl;
            }
            *reinterpret_cast<half8 *>(out_t + at) = h;
            *reinterpret_cast<half8 *>(out_t + out_plane + at) = l;
        }
        wave_exchange(); // the patch is written again
    }
}

template <typename T, Prod kProd, typename E>
void run_product(const OrthArgs &a, const OrthSteps &steps, char *ws, const OrthLayout &L, int k, hipStream_t st)
{
    constexpr size_t kRing = size_t(T::kStages) * 2 * (T::kM + T::kN) * kK * sizeof(f16);
    constexpr size_t kPatches = size_t(T::kWaves) * 16 * T::kHigh * T::kPatch * sizeof(float);
    constexpr size_t kLds = kRing > kPatches ? kRing : kPatches;
    static_assert(kLds <= 160 * 1024, "LDS of a CU");
    const auto at = [&](size_t bytes) { return reinterpret_cast<f16 *>(ws + bytes); };
    f16 *U = at(L.u[k & 1]), *V = at(L.v[k & 1]), *A = at(L.a), *B = at(L.b);
    const OrthStep &S = steps.step[k];
    const float next_sx = k + 1 < steps.count ? steps.step[k + 1].sx : 1.0f;
    const bool wide = a.rows <= a.cols;
    const int64_t plane = L.rows * L.cols, square = L.m * L.m;
    OrthProduct p = {};
    p.stride = int64_t(L.stride);
    p.lift = reinterpret_cast<const float *>(ws + L.lift);
    if constexpr (kProd == Prod::kGram || kProd == Prod::kPoly) {
        static_assert(T::kM == T::kN, "symmetric products");
        const int32_t mt = int32_t((L.m + T::kM - 1) / T::kM);
        p.tiles = mt * (mt + 1) / 2;
        p.P = p.Q = kProd == Prod::kPoly ? A : wide ? U : V;
        p.K = int32_t(kProd == Prod::kPoly ? L.m : L.n);
        p.p_plane = p.q_plane = kProd == Prod::kPoly ? square : plane;
        p.p_rows = p.q_rows = p.ld = p.ld_t = int32_t(L.m);
        p.out = p.out_t = kProd == Prod::kGram ? A : B;
        p.out_plane = square;
        p.old = A;
        if constexpr (kProd == Prod::kGram) {
            p.f_c = float(S.sa / (double(S.sx) * S.sx));
        } else {
            p.f_c = float(S.c * S.sb / (double(S.sa) * S.sa));
            p.f_old = float(S.b * S.sb / S.sa);
        }
    } else {
        const int32_t across = int32_t((L.cols + T::kN - 1) / T::kN);
        p.tiles = int32_t((L.rows + T::kM - 1) / T::kM) * across;
        p.across = 4 * across;
        p.per_four = uint32_t(((uint64_t(1) << 32) + p.across - 1) / p.across);
        p.P = wide ? B : U;
        p.Q = wide ? V : B;
        p.K = int32_t(L.m);
        p.p_plane = wide ? square : plane;
        p.q_plane = wide ? plane : square;
        p.p_rows = p.ld_t = int32_t(L.rows);
        p.q_rows = p.ld = int32_t(L.cols);
        p.out = at(L.u[(k + 1) & 1]);
        p.out_t = at(L.v[(k + 1) & 1]);
        p.out_plane = plane;
        p.old = U;
        p.f_c = float(next_sx / (double(S.sb) * S.sx));
        p.f_old = float(S.a * next_sx / S.sx);
        p.keep = a.keep;
        p.rate = a.rate;
        p.update = a.M != nullptr;
        p.rows = int32_t(a.rows);
        p.cols = int32_t(a.cols);
        p.W = a.W;
        p.w_batch = a.w_batch;
        p.w_stride = a.w_stride;
    }
    orth_product_kernel<T, kProd, E><<<dim3(uint32_t(p.tiles), 1, uint32_t(a.batch)), T::kThreads, kLds, st>>>(p);
}

// The tiles, each the best of several numbers of waves and buffers in the whole chain of products (whose operands come
// from other XCDs, where a probe that repeats one product finds them in its own L2).
using Tile32 = Tile<32, 32, 2, 2, 4>;
using Tile64 = Tile<64, 64, 2, 4, 3>;
using Tile64Several = Tile<64, 64, 2, 4, 2>; // less LDS: more blocks on a CU (1999 x 777 fp32: 40 us a step against 43)
using Tile96 = Tile<96, 96, 6, 2, 3>;
using Tile128 = Tile<128, 128, 2, 4, 2>;

// Which tile: the one whose busiest CU is done first.  Measured nanoseconds for a tile and slice of 64, of a CU that
// has one tile and of one that has several.
struct TileCost {
    int side;
    float one, several;
};
constexpr TileCost kTileCosts[] = {{32, 190, 131}, {64, 500, 361}, {96, 900, 820}, {128, 1390, 1110}};
struct TileChoice {
    int side;
    bool several; // tiles on a CU
};
TileChoice tile_of(bool symmetric, int64_t rows, int64_t cols, int64_t batch)
{
    TileChoice best = {0, false};
    float least = 0.0f;
    for (const TileCost &c : kTileCosts) {
        const int64_t down = (rows + c.side - 1) / c.side, across = (cols + c.side - 1) / c.side;
        const int64_t tiles = batch * (symmetric ? down * (down + 1) / 2 : down * across);
        const int64_t each = (tiles + kCus - 1) / kCus;
        const float cost = each <= 1 ? c.one : float(each) * c.several;
        if (best.side == 0 || cost < least) {
            best = {c.side, each > 1};
            least = cost;
        }
    }
    return best;
}

template <Prod kProd, typename E>
void run_tile(TileChoice choice, const OrthArgs &a, const OrthSteps &steps, char *ws, const OrthLayout &L, int k, hipStream_t st)
{
    const int tile = choice.side;
    if (tile == 32) return run_product<Tile32, kProd, E>(a, steps, ws, L, k, st);
    if (tile == 64 && choice.several) return run_product<Tile64Several, kProd, E>(a, steps, ws, L, k, st);
    if (tile == 64) return run_product<Tile64, kProd, E>(a, steps, ws, L, k, st);
    if (tile == 96) return run_product<Tile96, kProd, E>(a, steps, ws, L, k, st);
    run_product<Tile128, kProd, E>(a, steps, ws, L, k, st);
}

template <typename E>
void run_steps(const OrthArgs &a, const OrthSteps &steps, char *ws, const OrthLayout &L, hipStream_t st)
{
    const TileChoice square = tile_of(true, L.m, L.m, a.batch), full = tile_of(false, L.rows, L.cols, a.batch);
    for (int k = 0; k < steps.count; ++k) {
        run_tile<Prod::kGram, void>(square, a, steps, ws, L, k, st);
        run_tile<Prod::kPoly, void>(square, a, steps, ws, L, k, st);
        if (k + 1 < steps.count)
            run_tile<Prod::kApply, void>(full, a, steps, ws, L, k, st);
        else
            run_tile<Prod::kLast, E>(full, a, steps, ws, L, k, st);
    }
}

// ------------------------------------------------------------------ narrow matrices
// At most 64 directions (m <= 64).  Every step is a polynomial of A = X X^T, m x m, and these commute: with
// B = a I + b A + c A^2 the product of the steps is Q <- B Q, and the next A is B A B.  So U is read for one Gram
// matrix, the steps run on m x m matrices in one block's LDS, and Q is applied to U once: n enters twice, not
// 3 steps times.  In fewer than 64 bits A would lose the small singular values (their squares against the largest's;
// 1e-4 with 32); in fp64 on the matrix cores the result is off by its own rounding and 2e-8 at most (kNarrowNoise), and
// |U|^2 is A's trace.
// One launch where one block is quick with all of it; else one for the slices' Gram matrices and one in which every
// block adds them up in a fixed order, repeats the steps and applies Q to its columns.  Bound by the chain of products
// in one CU: a step takes 0.85 / 1.9 / 3.6 / 7.3 us for 16 / 32 / 48 / 64 directions (50: 6.5), of which the matrix core's 64 cycles
// a 16 x 16 x 4 product are 64 % for 64 directions (eleven tiles after one another on the fullest SIMD, 16 products each) and
// 58 % for 50 (13 each).  2 x 128 fp32 takes 7.9 us in all, 256 x 50 8.8 and 42.7.

typedef double double4v __attribute__((ext_vector_type(4)));

// A tile of 16 x 16: lane l holds rows l / 16 + 4 r of column l % 16
__device__ inline int tile_row(int r) { return lane_id() / 16 + 4 * r; }
__device__ inline int tile_col() { return lane_id() % 16; }

constexpr int narrow_waves(int tiles) { return tiles > 2 ? 16 : 8; }

// Tiles on and below the diagonal, in order of rows
template <int MT> struct Lower {
    static constexpr int kTiles = MT * (MT + 1) / 2;
    static constexpr int kParts = narrow_waves(MT) / kTiles; // waves that share the sum of a tile of the Gram matrix
    __device__ static int row(int t) { return t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3; }
    __device__ static int col(int t) { return t - row(t) * (row(t) + 1) / 2; }
};

enum class Narrow { kWhole, kGram, kApply };

struct NarrowSteps {
    int count;
    struct Step {
        double a, b, c;
    } step[kOrthMaxSteps];
};

template <int MT> constexpr int narrow_matrix() { return 16 * MT * (16 * MT + 2); } // doubles: 16 rows apart on all banks
template <int MT, Narrow kMode> constexpr size_t narrow_lds(int width)
{
    const size_t scratch = size_t(Lower<MT>::kParts - 1) * Lower<MT>::kTiles * 256, three = 3 * narrow_matrix<MT>();
    const size_t doubles = kMode == Narrow::kGram ? scratch : three > scratch ? three : scratch;
    return size_t(16 * MT) * (width + 4) * sizeof(float) + doubles * sizeof(double);
}

template <typename E, int MT, Narrow kMode>
__global__ __launch_bounds__(narrow_waves(MT) *kWave) void orth_narrow_kernel(OrthArgs a, NarrowSteps steps, char *ws, NarrowLayout L, int width, int shift)
{
    constexpr int kNarrowWaves = narrow_waves(MT), kNarrowBlock = kNarrowWaves * kWave;
    constexpr int kM = 16 * MT, kLd = kM + 2, kTiles = Lower<MT>::kTiles, kParts = Lower<MT>::kParts;
    extern __shared__ __align__(16) char s_mem[];
    __shared__ double s_sum[kNarrowWaves];
    float *U = reinterpret_cast<float *>(s_mem); // [kM][width + 4]: 16 rows by 4 columns on different banks
    const int ld_u = width + 4;
    double *mats = reinterpret_cast<double *>(U + kM * ld_u);
    double *A = mats, *B = A + narrow_matrix<MT>(), *Q = B + narrow_matrix<MT>();
    const int tid = threadIdx.x, lane = lane_id(), w = int(uniform(tid / kWave));
    const bool wide = a.rows <= a.cols;
    const int m = int(wide ? a.rows : a.cols);
    const int64_t n = wide ? a.cols : a.rows, z = blockIdx.y;
    double *partial = reinterpret_cast<double *>(ws + z * L.stride);

    // columns j0 .. of U into LDS, zeros around them; the momentum is updated where U is read first
    const auto load = [&](int64_t j0) {
        const int64_t g_i = wide ? a.g_stride : 1, g_j = wide ? 1 : a.g_stride; // steps along m and along n
        const int64_t m_i = wide ? a.m_stride : 1, m_j = wide ? 1 : a.m_stride;
        const E *G = static_cast<const E *>(a.G) + z * a.g_batch + j0 * g_j;
        float *M = a.M ? a.M + z * a.m_batch + j0 * m_j : nullptr;
        const int cols = int(n - j0 < width ? n - j0 : width);
        constexpr int kAtOnce = MT == 2 ? 16 : 8;
        for (int e0 = tid; e0 < kM * width; e0 += kAtOnce * kNarrowBlock) {
            float g[kAtOnce], mo[kAtOnce];
            int i[kAtOnce], j[kAtOnce];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                const int e = e0 + q * kNarrowBlock;
                i[q] = wide ? e >> shift : e % kM;
                j[q] = wide ? e & (width - 1) : e / kM;
                g[q] = i[q] < m && j[q] < cols ? float(G[i[q] * g_i + j[q] * g_j]) : 0.0f;
            }
            if (M) {
#pragma unroll
                for (int q = 0; q < kAtOnce; ++q) mo[q] = i[q] < m && j[q] < cols ? M[i[q] * m_i + j[q] * m_j] : 0.0f;
            }
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (M && kMode != Narrow::kApply) {
                    mo[q] = a.momentum * mo[q] + g[q];
                    if (i[q] < m && j[q] < cols) M[i[q] * m_i + j[q] * m_j] = mo[q];
                }
                if (e0 + q * kNarrowBlock < kM * width) U[i[q] * ld_u + j[q]] = M ? update_value(a, g[q], mo[q]) : g[q];
            }
        }
    };

    double scale = 0.0; // 1 / (|U| + eps)
    if constexpr (kMode != Narrow::kApply) {
        // the Gram matrix's lower tiles, a wave each, or several that share its columns
        double4v acc = {};
        const int t = w % kTiles, part = w / kTiles;
        const int ti = 16 * Lower<MT>::row(t), tj = 16 * Lower<MT>::col(t);
        for (int64_t j0 = int64_t(blockIdx.x) * width; j0 < n; j0 += int64_t(gridDim.x) * width) {
            load(j0);
            __syncthreads();
            const int cols = int(n - j0 < width ? n - j0 : width);
            constexpr int kDeep = 8; // 32 columns at a time
            for (int k0 = 4 * kDeep * part; part < kParts && k0 < cols; k0 += 4 * kDeep * kParts) {
                float x[kDeep], y[kDeep];
#pragma unroll
                for (int k = 0; k < kDeep; ++k) {
                    x[k] = U[(ti + lane % 16) * ld_u + k0 + 4 * k + lane / 16];
                    y[k] = U[(tj + lane % 16) * ld_u + k0 + 4 * k + lane / 16];
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < kDeep; ++k) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(double(x[k]), double(y[k]), acc, 0, 0, 0);
            }
            if constexpr (kMode == Narrow::kGram) __syncthreads();
        }
        if constexpr (kParts > 1) {
            if (part > 0 && part < kParts) {
#pragma unroll
                for (int r = 0; r < 4; ++r) mats[((part - 1) * kTiles + t) * 256 + r * kWave + lane] = acc[r];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int q = 0; q + 1 < kParts; ++q)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[r] += mats[(q * kTiles + t) * 256 + r * kWave + lane];
            }
        }
        if constexpr (kMode == Narrow::kGram) {
            if (part == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) partial[int64_t(blockIdx.x) * (kTiles * 256) + t * 256 + r * kWave + lane] = acc[r];
            }
            return;
        }
        double trace = 0.0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (part == 0 && ti + tile_row(r) == tj + tile_col()) trace += acc[r];
        trace = wave_sum(trace);
        if (lane == 0) s_sum[w] = trace;
        __syncthreads(); // mats is free too
        trace = 0.0;
        for (int q = 0; q < kTiles; ++q) trace += s_sum[q];
        scale = 1.0 / (sqrt(trace) + a.eps);
        if (part == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = ti + tile_row(r), col = tj + tile_col();
                A[row * kLd + col] = A[col * kLd + row] = acc[r] * (scale * scale);
            }
        }
        __syncthreads();
    } else {
        constexpr int kPer = (kTiles * 256 + kNarrowBlock - 1) / kNarrowBlock;
        double v[kPer] = {}, trace = 0.0;
        load(int64_t(blockIdx.x) * width); // on its way with the Gram matrices
#pragma unroll 8
        for (int q = 0; q < L.slices; ++q)
#pragma unroll
            for (int p = 0; p < kPer; ++p)
                if (tid + p * kNarrowBlock < kTiles * 256) v[p] += partial[int64_t(q) * (kTiles * 256) + tid + p * kNarrowBlock];
        // value e: tile e / 256, row of the tile (e / 64 % 4) and lane e % 64
        const auto place = [&](int e, int &row, int &col) {
            const int t = e / 256;
            row = 16 * Lower<MT>::row(t) + lane / 16 + 4 * (e / kWave % 4);
            col = 16 * Lower<MT>::col(t) + lane % 16;
        };
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            int row, col;
            place(tid + p * kNarrowBlock, row, col);
            if (tid + p * kNarrowBlock < kTiles * 256 && row == col) trace += v[p];
        }
        trace = wave_sum(trace);
        if (lane == 0) s_sum[w] = trace;
        __syncthreads();
        trace = 0.0;
        for (int q = 0; q < kNarrowWaves; ++q) trace += s_sum[q];
        scale = 1.0 / (sqrt(trace) + a.eps);
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            int row, col;
            place(tid + p * kNarrowBlock, row, col);
            if (tid + p * kNarrowBlock < kTiles * 256) A[row * kLd + col] = A[col * kLd + row] = v[p] * (scale * scale);
        }
        __syncthreads();
    }

    // Only the last tile can hold zeros behind the directions: of the groups of four terms all but three are sure to be
    // needed, and those that hold nothing are left out (256 x 50 fp32, momentum step: 51.5 us against 54.8)
    constexpr int kSure = kM / 4 - 3;
    // Lower tile t of a product of symmetric matrices, of which rows serve for columns
    const auto product = [&](const double *P, const double *R, int t) {
        const double *p = P + (16 * Lower<MT>::row(t) + lane % 16) * kLd + lane / 16;
        const double *q = R + (16 * Lower<MT>::col(t) + lane % 16) * kLd + lane / 16;
        // every operand is asked for before the first is used: a chain of products waits for LDS once
        double x[kM / 4], y[kM / 4];
#pragma unroll
        for (int k = 0; k < kM / 4; ++k) {
            x[k] = p[4 * k];
            y[k] = q[4 * k];
        }
        __builtin_amdgcn_sched_barrier(0);
        double4v acc = {};
#pragma unroll
        for (int k = 0; k < kM / 4; ++k)
            if (k < kSure || 4 * k < m) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[k], y[k], acc, 0, 0, 0);
        return acc;
    };
    // Both places of a pair take the one value below the diagonal: the products read rows for columns, so a difference
    // between the two, be it of a rounding, would grow (by 40 a step where A has no direction: 1.4 after 12 steps)
    const auto store = [&](double *P, int t, const double4v &v) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * Lower<MT>::row(t) + tile_row(r), col = 16 * Lower<MT>::col(t) + tile_col();
            if (row >= col) P[row * kLd + col] = P[col * kLd + row] = v[r];
        }
    };
    constexpr int kOne = (kTiles + kNarrowWaves - 1) / kNarrowWaves, kTwo = (2 * kTiles + kNarrowWaves - 1) / kNarrowWaves;
    for (int s = 0; s < steps.count; ++s) {
        const NarrowSteps::Step &S = steps.step[s];
        const bool last = s + 1 == steps.count;
        // B = a I + b A + c A^2, and the first Q
#pragma unroll
        for (int q = 0; q < kOne; ++q) {
            const int t = w + q * kNarrowWaves;
            if (t >= kTiles) continue;
            double4v v = product(A, A, t);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * Lower<MT>::row(t) + tile_row(r), col = 16 * Lower<MT>::col(t) + tile_col();
                v[r] = S.b * A[row * kLd + col] + S.c * v[r] + (row == col ? S.a : 0.0);
            }
            store(B, t, v);
            if (s == 0) store(Q, t, v);
        }
        __syncthreads();
        // B Q and A B at once, each in its factor's place when everybody has read it
        double4v v[kTwo];
        const int items = (last ? 0 : kTiles) + (s == 0 ? 0 : kTiles), from = s == 0 ? kTiles : 0;
#pragma unroll
        for (int q = 0; q < kTwo; ++q) {
            const int t = from + w + q * kNarrowWaves;
            if (t < from + items) v[q] = t < kTiles ? product(B, Q, t) : product(A, B, t - kTiles);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kTwo; ++q) {
            const int t = from + w + q * kNarrowWaves;
            if (t < from + items) store(t < kTiles ? Q : A, t < kTiles ? t : t - kTiles, v[q]);
        }
        __syncthreads();
        if (last) break;
        // the next A = (A B) B
#pragma unroll
        for (int q = 0; q < kOne; ++q)
            if (w + q * kNarrowWaves < kTiles) v[q] = product(A, B, w + q * kNarrowWaves);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kOne; ++q)
            if (w + q * kNarrowWaves < kTiles) store(A, w + q * kNarrowWaves, v[q]);
        __syncthreads();
    }

    // X = Q U / (|U| + eps), 16 columns a wave at a time
    const int64_t w_i = wide ? a.w_stride : 1, w_j = wide ? 1 : a.w_stride;
    for (int64_t j0 = int64_t(blockIdx.x) * width; j0 < n; j0 += int64_t(gridDim.x) * width) {
        if (kMode == Narrow::kApply && j0 != int64_t(blockIdx.x) * width) { // the first columns are there
            __syncthreads();
            load(j0);
            __syncthreads();
        }
        const int cols = int(n - j0 < width ? n - j0 : width);
        E *out = static_cast<E *>(a.W) + z * a.w_batch + j0 * w_j;
        for (int jt = 16 * w; jt < cols; jt += 16 * kNarrowWaves) {
            double u[kM / 4];
#pragma unroll
            for (int k = 0; k < kM / 4; ++k) u[k] = double(U[(4 * k + lane / 16) * ld_u + jt + lane % 16]);
            const int j = jt + lane % 16;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const double *p = Q + (16 * i + lane % 16) * kLd + lane / 16;
                double x[kM / 4];
#pragma unroll
                for (int k = 0; k < kM / 4; ++k) x[k] = p[4 * k];
                __builtin_amdgcn_sched_barrier(0);
                double4v acc = {};
#pragma unroll
                for (int k = 0; k < kM / 4; ++k)
                    if (k < kSure || 4 * k < m) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[k], u[k], acc, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + tile_row(r);
                    if (row >= m || j >= cols) continue;
                    E *o = out + row * w_i + j * w_j;
                    const float x = float(acc[r] * scale);
                    *o = E(a.M ? a.keep * float(*o) - a.rate * x : x);
                }
            }
        }
    }
}

// ------------------------------------------------------------------ narrow matrices, many steps
// Stepping on A alone loses the directions that X lacks: their eigenvalues are zero but for rounding, of either sign,
// grow by a^2 a step, and below zero without end.  Where that would show (kNarrowNoise) X itself is stepped on, in fp64:
// X <- a X + (b A + c A^2) X with A = X X^T formed from X each time, whose errors grow by a and stay bounded, as in the
// formula.  Two launches a step, by plain products: 32 steps of 32 x 100 fp32 take 0.75 ms, of 64 x 4096 1.7.
// Every row's sums run in one order, so that equal rows stay equal.
constexpr int kDirectLd = kDirect + 1;
constexpr size_t kDirectLds = 2 * size_t(kDirect) * kDirectLd * sizeof(double);

// X = U / (|U| + eps)
template <typename E>
__global__ __launch_bounds__(256) void orth_direct_start_kernel(OrthArgs a, char *ws, DirectLayout L, int norm_blocks)
{
    const int64_t z = blockIdx.y;
    char *base = ws + z * L.stride;
    const double *part = reinterpret_cast<const double *>(base + L.norm);
    double sq = 0.0;
    for (int k = lane_id(); k < norm_blocks; k += kWave) sq += part[k];
    const double scale = 1.0 / (sqrt(wave_sum(sq)) + a.eps);
    double *X = reinterpret_cast<double *>(base + L.x);
    const bool wide = a.rows <= a.cols;
    const uint32_t cols = uint32_t(a.cols), total = uint32_t(a.rows) * cols; // <= 2^22
    for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < total; e += gridDim.x * 256) {
        const uint32_t r = e / cols, c = e - r * cols;
        const float g = float(static_cast<const E *>(a.G)[z * a.g_batch + r * a.g_stride + c]);
        const float m = a.M ? a.M[z * a.m_batch + r * a.m_stride + c] : 0.0f;
        X[wide ? int64_t(e) : c * L.n + r] = double(update_value(a, g, m)) * scale;
    }
}

// columns j0 .. j0 + kDirect of X into LDS, zeros around them
__device__ inline void direct_load(const double *X, const DirectLayout &L, int64_t j0, double *s_x)
{
    for (int e = threadIdx.x; e < kDirect * kDirect; e += 256) {
        const int i = e / kDirect, j = e % kDirect;
        s_x[i * kDirectLd + j] = i < L.m && j0 + j < L.n ? X[i * L.n + j0 + j] : 0.0;
    }
}

// Partial Gram matrices: a thread has rows ty + 16 p and columns tx + 16 q of one
__global__ __launch_bounds__(256) void orth_direct_gram_kernel(char *ws, DirectLayout L)
{
    extern __shared__ __align__(16) char s_mem[];
    double *s_x = reinterpret_cast<double *>(s_mem);
    char *base = ws + int64_t(blockIdx.y) * L.stride;
    const double *X = reinterpret_cast<const double *>(base + L.x);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    double acc[4][4] = {};
    for (int64_t j0 = int64_t(blockIdx.x) * kDirect; j0 < L.n; j0 += int64_t(gridDim.x) * kDirect) {
        __syncthreads();
        direct_load(X, L, j0, s_x);
        __syncthreads();
        for (int k = 0; k < kDirect; ++k)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    acc[p][q] = fma(s_x[(ty + 16 * p) * kDirectLd + k], s_x[(tx + 16 * q) * kDirectLd + k], acc[p][q]);
    }
    double *part = reinterpret_cast<double *>(base + L.gram) + int64_t(blockIdx.x) * L.m * L.m;
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (ty + 16 * p < L.m && tx + 16 * q < L.m) part[(ty + 16 * p) * L.m + tx + 16 * q] = acc[p][q];
}

// A step: every block adds up A, forms b A + c A^2 and takes its columns of X on; the last writes the output
template <typename E>
__global__ __launch_bounds__(256) void orth_direct_step_kernel(OrthArgs a, char *ws, DirectLayout L, NarrowSteps::Step S, bool last)
{
    extern __shared__ __align__(16) char s_mem[];
    double *s_a = reinterpret_cast<double *>(s_mem), *s_x = s_a + kDirect * kDirectLd;
    const int64_t z = blockIdx.y;
    char *base = ws + z * L.stride;
    double *X = reinterpret_cast<double *>(base + L.x);
    const double *part = reinterpret_cast<const double *>(base + L.gram);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int e = threadIdx.x; e < kDirect * kDirect; e += 256) {
        const int i = e / kDirect, j = e % kDirect;
        double s = 0.0;
        if (i < L.m && j < L.m)
#pragma unroll 8
            for (int k = 0; k < L.slices; ++k) s += part[(int64_t(k) * L.m + i) * L.m + j];
        s_a[i * kDirectLd + j] = s;
    }
    __syncthreads();
    double acc[4][4] = {};
    for (int k = 0; k < L.m; ++k)
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc[p][q] = fma(s_a[(ty + 16 * p) * kDirectLd + k], s_a[(tx + 16 * q) * kDirectLd + k], acc[p][q]);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            double &v = s_a[(ty + 16 * p) * kDirectLd + tx + 16 * q];
            v = S.b * v + S.c * acc[p][q];
        }
    const bool wide = a.rows <= a.cols;
    const int64_t w_i = wide ? a.w_stride : 1, w_j = wide ? 1 : a.w_stride;
    for (int64_t j0 = int64_t(blockIdx.x) * kDirect; j0 < L.n; j0 += int64_t(gridDim.x) * kDirect) {
        __syncthreads();
        direct_load(X, L, j0, s_x);
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[p][q] = S.a * s_x[(ty + 16 * p) * kDirectLd + tx + 16 * q];
        for (int k = 0; k < L.m; ++k)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    acc[p][q] = fma(s_a[(ty + 16 * p) * kDirectLd + k], s_x[k * kDirectLd + tx + 16 * q], acc[p][q]);
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = ty + 16 * p;
                const int64_t j = j0 + tx + 16 * q;
                if (i >= L.m || j >= L.n) continue;
                if (!last) {
                    X[i * L.n + j] = acc[p][q];
                    continue;
                }
                E *o = static_cast<E *>(a.W) + z * a.w_batch + i * w_i + j * w_j;
                const float x = float(acc[p][q]);
                *o = E(a.M ? a.keep * float(*o) - a.rate * x : x);
            }
    }
}

int log2_of(int x)
{
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

template <typename E, int MT> void run_narrow(const OrthArgs &a, const NarrowSteps &steps, char *ws, const NarrowLayout &L, hipStream_t st)
{
    constexpr int kBlock = narrow_waves(MT) * kWave;
    const int shift = log2_of(L.width);
    const uint32_t z = uint32_t(a.batch);
    if (L.slices == 0) {
        orth_narrow_kernel<E, MT, Narrow::kWhole>
            <<<dim3(1, z), kBlock, narrow_lds<MT, Narrow::kWhole>(L.width), st>>>(a, steps, ws, L, L.width, shift);
        return;
    }
    orth_narrow_kernel<E, MT, Narrow::kGram>
        <<<dim3(uint32_t(L.slices), z), kBlock, narrow_lds<MT, Narrow::kGram>(L.width), st>>>(a, steps, ws, L, L.width, shift);
    // each block repeats the steps: no more blocks than find a CU free
    const int64_t n = a.rows > a.cols ? a.rows : a.cols, chunks = (n + L.width - 1) / L.width;
    const int64_t most = a.batch < kCus ? kCus / a.batch : 1, blocks = chunks < most ? chunks : most;
    orth_narrow_kernel<E, MT, Narrow::kApply>
        <<<dim3(uint32_t(blocks), z), kBlock, narrow_lds<MT, Narrow::kApply>(L.width), st>>>(a, steps, ws, L, L.width, shift);
}

} // namespace

int norm_blocks_of(int64_t rows, int64_t cols)
{
    const int64_t want = (rows * cols + 2047) / 2048; // 8 values a thread
    return int(want < kOrthNormBlocks ? want : kOrthNormBlocks);
}

NarrowLayout make_narrow_layout(int64_t rows, int64_t cols)
{
    // one block as long as its Gram matrix and its product with Q take 6 us or less, the cost of a second launch
    static_assert(narrow_lds<1, Narrow::kWhole>(2048) <= 160 * 1024 && narrow_lds<2, Narrow::kWhole>(512) <= 160 * 1024 &&
                      narrow_lds<3, Narrow::kWhole>(256) <= 160 * 1024 && narrow_lds<4, Narrow::kWhole>(128) <= 160 * 1024 &&
                      narrow_lds<4, Narrow::kGram>(kNarrowSlice) <= 160 * 1024,
                  "LDS of a CU");
    constexpr int kWhole[4] = {2048, 512, 256, 128};
    NarrowLayout L;
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    L.tiles = int((m + 15) / 16);
    L.slices = 0;
    L.width = 64;
    while (L.width < n && L.width < kWhole[L.tiles - 1]) L.width *= 2;
    if (L.width < n) {
        L.width = kNarrowSlice;
        const int64_t chunks = (n + L.width - 1) / L.width;
        L.slices = int(chunks < kNarrowSlices ? chunks : kNarrowSlices);
    }
    L.stride = size_t(L.slices > 0 ? L.slices : 1) * (L.tiles * (L.tiles + 1) / 2) * 256 * sizeof(double);
    return L;
}

OrthLayout make_orth_layout(int64_t rows, int64_t cols)
{
    OrthLayout L;
    const auto pad = [&](int64_t x) { return (x + kK - 1) / kK * kK; }; // every row is whole slices
    L.rows = pad(rows);
    L.cols = pad(cols);
    L.m = L.rows < L.cols ? L.rows : L.cols;
    L.n = L.rows < L.cols ? L.cols : L.rows;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const size_t planes = 2 * sizeof(f16);
    for (int k = 0; k < 2; ++k) {
        L.u[k] = take(planes * L.rows * L.cols);
        L.v[k] = take(planes * L.rows * L.cols);
    }
    L.a = take(planes * L.m * L.m);
    L.b = take(planes * L.m * L.m);
    L.norm = take(sizeof(double) * kOrthNormBlocks);
    L.lift = take(sizeof(float));
    L.stride = at;
    return L;
}

DirectLayout make_direct_layout(int64_t rows, int64_t cols)
{
    DirectLayout L;
    L.m = int(rows < cols ? rows : cols);
    L.n = rows < cols ? cols : rows;
    const int64_t chunks = (L.n + kDirect - 1) / kDirect;
    L.slices = int(chunks < kDirectSlices ? chunks : kDirectSlices);
    const auto whole = [](size_t doubles) { return (doubles * sizeof(double) + 255) / 256 * 256; };
    L.norm = 0;
    L.gram = whole(kOrthNormBlocks);
    L.x = L.gram + whole(size_t(L.slices) * L.m * L.m);
    L.stride = L.x + whole(size_t(L.m) * L.n);
    return L;
}

size_t orth_workspace(int64_t rows, int64_t cols)
{
    if (!orth_narrow(rows, cols)) return make_orth_layout(rows, cols).stride;
    const size_t few = make_narrow_layout(rows, cols).stride, many = make_direct_layout(rows, cols).stride;
    return few > many ? few : many; // how many steps there will be is not asked
}

namespace {

// rows and matrices start on 16 bytes
bool vectors(const void *p, int64_t stride, int64_t batch_stride, int64_t batch, int bytes)
{
    return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(stride * bytes) | uintptr_t(batch > 1 ? batch_stride * bytes : 0)) & 15u) == 0;
}

template <typename E> void run_wide(const OrthArgs &a, const OrthSteps &steps, char *ws, hipStream_t st)
{
    const OrthLayout L = make_orth_layout(a.rows, a.cols);
    const int norm_blocks = norm_blocks_of(a.rows, a.cols);
    // matrices without gaps are rows of rows x cols values there, whose 16-byte accesses any length of row allows
    // (1999 x 777 fp32 with its momentum 5.8 us, by rows 11.9)
    OrthArgs flat = a;
    if (a.g_stride == a.cols && (!a.M || a.m_stride == a.cols)) {
        flat.cols = flat.g_stride = flat.m_stride = a.rows * a.cols;
        flat.rows = 1;
        flat.g_vec = vectors(a.G, 0, a.g_batch, a.batch, elem_bytes(a.type));
        flat.m_vec = vectors(a.M, 0, a.m_batch, a.batch, 4);
    }
    orth_norm_kernel<E><<<dim3(norm_blocks, uint32_t(a.batch)), 256, 0, st>>>(flat, ws, int64_t(L.stride), L.norm);
    orth_planes_kernel<E><<<dim3(uint32_t(L.cols / kT), uint32_t(L.rows / kT), uint32_t(a.batch)), 256, 0, st>>>(
        a, ws, L, norm_blocks, steps.step[0].sx, steps.reach);
    run_steps<E>(a, steps, ws, L, st);
}

template <typename E> void run_direct(const OrthArgs &a, const OrthSteps &steps, char *ws, hipStream_t st)
{
    const DirectLayout L = make_direct_layout(a.rows, a.cols);
    const uint32_t z = uint32_t(a.batch);
    // by rows, whatever lies between them: the norm's sum has one order, and many steps would show another
    const int norm_blocks = norm_blocks_of(a.rows, a.cols);
    orth_norm_kernel<E><<<dim3(norm_blocks, z), 256, 0, st>>>(a, ws, int64_t(L.stride), L.norm);
    orth_direct_start_kernel<E><<<dim3(uint32_t((a.rows * a.cols + 1023) / 1024), z), 256, 0, st>>>(a, ws, L, norm_blocks);
    const int64_t chunks = (L.n + kDirect - 1) / kDirect, blocks = chunks < kCus ? chunks : kCus;
    for (int k = 0; k < steps.count; ++k) {
        const NarrowSteps::Step S = {steps.step[k].a, steps.step[k].b, steps.step[k].c};
        orth_direct_gram_kernel<<<dim3(uint32_t(L.slices), z), 256, kDirectLds / 2, st>>>(ws, L);
        orth_direct_step_kernel<E><<<dim3(uint32_t(blocks), z), 256, kDirectLds, st>>>(a, ws, L, S, k + 1 == steps.count);
    }
}

template <typename E> void run_type(const OrthArgs &a, const OrthSteps &steps, char *ws, hipStream_t st)
{
    if (orth_narrow(a.rows, a.cols) && steps.noise > kNarrowNoise) return run_direct<E>(a, steps, ws, st);
    if (orth_narrow(a.rows, a.cols)) {
        const NarrowLayout L = make_narrow_layout(a.rows, a.cols);
        NarrowSteps narrow;
        narrow.count = steps.count;
        for (int k = 0; k < steps.count; ++k) narrow.step[k] = {steps.step[k].a, steps.step[k].b, steps.step[k].c};
        if (L.tiles == 1) return run_narrow<E, 1>(a, narrow, ws, L, st);
        if (L.tiles == 2) return run_narrow<E, 2>(a, narrow, ws, L, st);
        if (L.tiles == 3) return run_narrow<E, 3>(a, narrow, ws, L, st);
        return run_narrow<E, 4>(a, narrow, ws, L, st);
    }
    run_wide<E>(a, steps, ws, st);
}

} // namespace

void launch_orthogonalise(const OrthArgs &args, const OrthSteps &steps, void *workspace, hipStream_t st)
{
    if (args.batch == 0) return;
    OrthArgs a = args;
    a.g_vec = vectors(a.G, a.g_stride, a.g_batch, a.batch, elem_bytes(a.type));
    a.m_vec = vectors(a.M, a.m_stride, a.m_batch, a.batch, 4);
    char *ws = static_cast<char *>(workspace);
    if (a.type == Elem::kF32)
        run_type<float>(a, steps, ws, st);
    else if (a.type == Elem::kF16)
        run_type<f16>(a, steps, ws, st);
    else
        run_type<bf16>(a, steps, ws, st);
}

} // namespace bht
