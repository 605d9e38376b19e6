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
// factor of a each step against the largest, so a X must come from both halves;
// B X may come from rounded operands when the output has 8 bits (bf16) and the
// matrix more than kOrthOneProduct directions: the error before the output's
// rounding is then about 1e-3 (gaussian, decaying and nearly low-rank matrices).
// Otherwise each product is three, high by high and the two mixed ones, and as
// exact as products in 32 bits.
#include <type_traits>

#include "map.hpp"

namespace bht {
namespace {

typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kT = kOrthTile;
constexpr int kK = 64;          // depth of a staged slice: 128 bytes a row
constexpr int kProdBlock = 256; // 4 waves

__device__ inline float load_elem(const void *p, Elem t, int64_t i)
{
    if (t == Elem::kF32) return static_cast<const float *>(p)[i];
    if (t == Elem::kF16) return float(static_cast<const f16 *>(p)[i]);
    return float(static_cast<const bf16 *>(p)[i]);
}
__device__ inline void store_elem(void *p, Elem t, int64_t i, float v)
{
    if (t == Elem::kF32)
        static_cast<float *>(p)[i] = v;
    else if (t == Elem::kF16)
        static_cast<f16 *>(p)[i] = f16(v);
    else
        static_cast<bf16 *>(p)[i] = bf16(v);
}

// ------------------------------------------------------------------ norm and planes
__device__ inline float update_value(const OrthArgs &a, float g, float m)
{
    return a.M ? (a.nesterov != 0.0f ? g + a.momentum * m : m) : g;
}

// The momentum's update, and partial sums of U's squares: fp64, in a fixed order.
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs a, char *ws, OrthLayout L)
{
    __shared__ double s_w[256 / kWave];
    const int64_t z = blockIdx.y;
    double sum = 0.0;
    const int64_t total = a.rows * a.cols;
    const int64_t per = (total + gridDim.x - 1) / gridDim.x; // a contiguous range of elements each
    const int64_t lo = blockIdx.x * per, hi = lo + per < total ? lo + per : total;
    for (int64_t e = lo + threadIdx.x; e < hi; e += 256) {
        const int64_t r = e / a.cols, c = e - r * a.cols;
        float g = load_elem(a.G, a.type, z * a.g_batch + r * a.g_stride + c), m = 0.0f;
        if (a.M) {
            float *M = a.M + z * a.m_batch + r * a.m_stride + c;
            m = a.momentum * *M + g;
            *M = m;
        }
        const double u = double(update_value(a, g, m));
        sum += u * u;
    }
    sum = wave_sum(sum);
    if (lane_id() == 0) s_w[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < 256 / kWave; ++w) t += s_w[w];
        reinterpret_cast<double *>(ws + z * L.stride + L.norm)[blockIdx.x] = t;
    }
}

__device__ inline void split(float v, f16 &h, f16 &l)
{
    h = f16(v);
    l = f16(v - float(h));
}

// U / (|U| + eps) in planes, in both orientations, zeros in the padding
__global__ __launch_bounds__(256) void orth_planes_kernel(OrthArgs a, char *ws, OrthLayout L, int norm_blocks)
{
    __shared__ f16 s_t[2][kT][kT + 2];
    const int64_t z = blockIdx.z, r0 = int64_t(blockIdx.y) * kT, c0 = int64_t(blockIdx.x) * kT;
    char *base = ws + z * L.stride;
    const double *part = reinterpret_cast<const double *>(base + L.norm);
    double sq = 0.0;
    for (int k = lane_id(); k < norm_blocks; k += kWave) sq += part[k];
    sq = wave_sum(sq);
    const double scale = double(a.step[0].sx) / (sqrt(sq) + a.eps);
    f16 *uh = reinterpret_cast<f16 *>(base + L.u[0]), *ul = uh + L.rows * L.cols;
    f16 *vh = reinterpret_cast<f16 *>(base + L.v[0]), *vl = vh + L.rows * L.cols;
    for (int e = threadIdx.x; e < kT * kT; e += 256) {
        const int i = e / kT, j = e % kT;
        const int64_t r = r0 + i, c = c0 + j;
        float v = 0.0f;
        if (r < a.rows && c < a.cols) {
            const float g = load_elem(a.G, a.type, z * a.g_batch + r * a.g_stride + c);
            const float m = a.M ? a.M[z * a.m_batch + r * a.m_stride + c] : 0.0f;
            v = float(double(update_value(a, g, m)) * scale);
        }
        f16 h, l;
        split(v, h, l);
        uh[r * L.cols + c] = h;
        ul[r * L.cols + c] = l;
        s_t[0][j][i] = h;
        s_t[1][j][i] = l;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kT * kT; e += 256) {
        const int j = e / kT, i = e % kT;
        vh[(c0 + j) * L.rows + r0 + i] = s_t[0][j][i];
        vl[(c0 + j) * L.rows + r0 + i] = s_t[1][j][i];
    }
}

// ------------------------------------------------------------------ products
enum class Prod { kGram, kPoly, kApply, kLast };

// One tile of C = P Q^T, P and Q row-major with K values a row.  Operands are staged in
// LDS by loads that write it directly; a row's eight 16-byte pieces are stored in
// an order that depends on the row (piece c of row r in place c ^ (r % 8)), so
// that the lanes of a fragment read, which take the same piece of 32 rows, fall on
// different banks.
template <bool kSplit> struct Staged {
    f16 p[kSplit ? 2 : 1][kT * kK];
    f16 q[kSplit ? 2 : 1][kT * kK];
};
template <bool kSplit> union alignas(16) Shared {
    Staged<kSplit> in;
    float out[kT][kT + 1];
};

__device__ inline void stage(const f16 *src, int64_t ld, f16 *dst)
{
    const int w = threadIdx.x / kWave, lane = lane_id();
    const int r = lane / 8, piece = (lane % 8) ^ r;
#pragma unroll
    for (int k = 0; k < kT / 32; ++k) {
        const int row = (k * 4 + w) * 8;
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void *)(src + (row + r) * ld + piece * 8),
            (__attribute__((address_space(3))) void *)(dst + row * kK), 16, 0, 0);
    }
}

__device__ inline half8 fragment(const f16 *tile, int row, int piece)
{
    return *reinterpret_cast<const half8 *>(tile + row * kK + ((piece ^ (row & 7)) * 8));
}

template <bool kSplit, Prod kProd>
__global__ __launch_bounds__(kProdBlock) void orth_product_kernel(OrthArgs a, char *ws, OrthLayout L, int k)
{
    __shared__ Shared<kSplit> s;
    const OrthStep &S = a.step[k];
    const bool wide = a.rows <= a.cols;
    char *base = ws + int64_t(blockIdx.z) * L.stride;
    const int64_t plane = L.rows * L.cols, square = L.m * L.m;
    f16 *U = reinterpret_cast<f16 *>(base + L.u[k & 1]), *V = reinterpret_cast<f16 *>(base + L.v[k & 1]);
    f16 *A = reinterpret_cast<f16 *>(base + L.a), *B = reinterpret_cast<f16 *>(base + L.b);
    int64_t bi, bj;
    const f16 *P, *Q;
    int64_t K, p_plane, q_plane;
    if constexpr (kProd == Prod::kGram || kProd == Prod::kPoly) {
        // tiles on and below the diagonal, row by row
        const int t = blockIdx.x;
        bi = int64_t((sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
        while (bi * (bi + 1) / 2 > t) --bi;
        bj = t - bi * (bi + 1) / 2;
        if constexpr (kProd == Prod::kGram) {
            P = Q = wide ? U : V;
            K = L.n;
            p_plane = q_plane = plane;
        } else {
            P = Q = A;
            K = L.m;
            p_plane = q_plane = square;
        }
    } else {
        bi = blockIdx.y;
        bj = blockIdx.x;
        K = L.m;
        P = wide ? B : U;
        Q = wide ? V : B;
        p_plane = wide ? square : plane;
        q_plane = wide ? plane : square;
    }
    P += bi * kT * K;
    Q += bj * kT * K;
    const int w = threadIdx.x / kWave, lane = lane_id();
    const int wi = (w / 2) * 32, wj = (w % 2) * 32;
    float16v acc = {};
    for (int64_t k0 = 0; k0 < K; k0 += kK) {
        __syncthreads();
        stage(P + k0, K, s.in.p[0]);
        stage(Q + k0, K, s.in.q[0]);
        if constexpr (kSplit) {
            stage(P + p_plane + k0, K, s.in.p[1]);
            stage(Q + q_plane + k0, K, s.in.q[1]);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // the staged slice is in LDS
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kK / 16; ++kk) {
            const int piece = kk * 2 + lane / 32;
            const half8 ph = fragment(s.in.p[0], wi + lane % 32, piece), qh = fragment(s.in.q[0], wj + lane % 32, piece);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
            if constexpr (kSplit) {
                const half8 pl = fragment(s.in.p[1], wi + lane % 32, piece), ql = fragment(s.in.q[1], wj + lane % 32, piece);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 16; ++r) s.out[wi + 8 * (r / 4) + 4 * (lane / 32) + r % 4][wj + lane % 32] = acc[r];
    __syncthreads();

    const int64_t r0 = bi * kT, c0 = bj * kT;
    // values in the tile's own orientation
    f16 *out_h = nullptr;
    int64_t ld = 0, out_plane = 0;
    if constexpr (kProd == Prod::kGram) {
        out_h = A;
        ld = L.m;
        out_plane = square;
    } else if constexpr (kProd == Prod::kPoly) {
        out_h = B;
        ld = L.m;
        out_plane = square;
    } else if constexpr (kProd == Prod::kApply) {
        out_h = reinterpret_cast<f16 *>(base + L.u[(k + 1) & 1]);
        ld = L.cols;
        out_plane = plane;
    }
    const float xs = kProd == Prod::kApply ? a.step[k + 1].sx / S.sx : 1.0f / S.sx;
    for (int e = threadIdx.x; e < kT * kT; e += kProdBlock) {
        const int i = e / kT, j = e % kT;
        const int64_t r = r0 + i, c = c0 + j;
        float v = s.out[i][j];
        if constexpr (kProd == Prod::kGram) {
            v *= S.sa / (S.sx * S.sx);
        } else if constexpr (kProd == Prod::kPoly) {
            const float av = float(A[r * L.m + c]) + float(A[square + r * L.m + c]);
            v = av * (S.b * S.sb / S.sa) + v * (S.c * S.sb / (S.sa * S.sa));
        } else {
            const float x = float(U[r * L.cols + c]) + float(U[plane + r * L.cols + c]);
            v = (S.a * x + v / S.sb) * xs;
        }
        if constexpr (kProd == Prod::kLast) {
            if (r < a.rows && c < a.cols) {
                const int64_t at = int64_t(blockIdx.z) * a.w_batch + r * a.w_stride + c;
                if (a.M) v = a.keep * load_elem(a.W, a.type, at) - a.rate * v;
                store_elem(a.W, a.type, at, v);
            }
        } else {
            f16 h, l;
            split(v, h, l);
            out_h[r * ld + c] = h;
            out_h[out_plane + r * ld + c] = l;
            s.out[i][j] = v;
        }
    }
    if constexpr (kProd != Prod::kLast) {
        if (kProd != Prod::kApply && bi == bj) return;
        __syncthreads();
        f16 *t_h = kProd == Prod::kApply ? reinterpret_cast<f16 *>(base + L.v[(k + 1) & 1]) : out_h;
        const int64_t t_ld = kProd == Prod::kApply ? L.rows : L.m;
        for (int e = threadIdx.x; e < kT * kT; e += kProdBlock) {
            const int j = e / kT, i = e % kT;
            f16 h, l;
            split(s.out[i][j], h, l);
            t_h[(c0 + j) * t_ld + r0 + i] = h;
            t_h[out_plane + (c0 + j) * t_ld + r0 + i] = l;
        }
    }
}

template <bool kSplit> void run_steps(const OrthArgs &a, char *ws, const OrthLayout &L, hipStream_t st)
{
    const uint32_t mt = uint32_t(L.m / kT), tri = mt * (mt + 1) / 2, z = uint32_t(a.batch);
    const dim3 square(tri, 1, z), full(uint32_t(L.cols / kT), uint32_t(L.rows / kT), z);
    for (int k = 0; k < a.steps; ++k) {
        orth_product_kernel<kSplit, Prod::kGram><<<square, kProdBlock, 0, st>>>(a, ws, L, k);
        orth_product_kernel<kSplit, Prod::kPoly><<<square, kProdBlock, 0, st>>>(a, ws, L, k);
        if (k + 1 < a.steps)
            orth_product_kernel<kSplit, Prod::kApply><<<full, kProdBlock, 0, st>>>(a, ws, L, k);
        else
            orth_product_kernel<kSplit, Prod::kLast><<<full, kProdBlock, 0, st>>>(a, ws, L, k);
    }
}

} // namespace

OrthLayout make_orth_layout(int64_t rows, int64_t cols)
{
    OrthLayout L;
    const auto pad = [](int64_t x) { return (x + kT - 1) / kT * kT; };
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
    L.stride = at;
    return L;
}

void launch_orthogonalise(const OrthArgs &a, void *workspace, hipStream_t st)
{
    if (a.batch == 0) return;
    char *ws = static_cast<char *>(workspace);
    const OrthLayout L = make_orth_layout(a.rows, a.cols);
    const int64_t want = (a.rows * a.cols + 4095) / 4096;
    const int norm_blocks = int(want < kOrthNormBlocks ? want : kOrthNormBlocks);
    orth_norm_kernel<<<dim3(norm_blocks, uint32_t(a.batch)), 256, 0, st>>>(a, ws, L);
    orth_planes_kernel<<<dim3(uint32_t(L.cols / kT), uint32_t(L.rows / kT), uint32_t(a.batch)), 256, 0, st>>>(a, ws, L, norm_blocks);
    if (orth_split(a.type, a.rows, a.cols))
        run_steps<true>(a, ws, L, st);
    else
        run_steps<false>(a, ws, L, st);
}

} // namespace bht
