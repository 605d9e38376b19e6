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
// matrix is not narrow: the error before the output's
// rounding is then about 1e-3 (gaussian, decaying and nearly low-rank matrices).
// Otherwise each product is three, high by high and the two mixed ones, as exact
// as products in 32 bits, and a I is part of B.
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
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs a, char *ws, int64_t ws_stride, size_t at)
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
        reinterpret_cast<double *>(ws + z * ws_stride + at)[blockIdx.x] = t;
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
            if (kSplit && r == c) v += S.a * S.sb;
        } else {
            v *= 1.0f / S.sb;
            if constexpr (!kSplit) v += S.a * (float(U[r * L.cols + c]) + float(U[plane + r * L.cols + c]));
            v *= xs;
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

// ------------------------------------------------------------------ narrow matrices
// At most 64 directions (m <= 64).  X lives in LDS, as fp16 halves and in both orientations: rows of X for the
// Gram matrix (the sum runs along n), rows of X^T for B X (along m).  A matrix whose X fits one block's LDS takes
// one launch for everything: all steps between two reads and one write.  A longer one is cut into slices of
// kSlice columns, a block each, and takes one launch a step: every block adds up the slices' Gram matrices (or
// reads their sum, made by a launch of its own, where slices are many), forms B = a I + b A + c A^2 itself, applies
// it to its slice and leaves the new X's partial Gram matrix for the next launch.  The sums are in a fixed order.
constexpr int kNarrowBlock = 512; // 8 waves
constexpr int kSlice = 128;
constexpr int kSliceSum = 16;     // slices whose Gram matrices every block adds up itself

typedef f16 half4 __attribute__((ext_vector_type(4)));

// place of 8-value piece p of row r in planes of ld values a row (32 or a multiple of 64): the same piece of
// consecutive rows on different banks
__device__ inline int piece_at(int r, int p, int ld)
{
    return r * ld + ((ld == 32 ? p ^ ((r >> 2) & 3) : p ^ (r & 7)) * 8);
}

struct Planes {
    f16 *h, *l;
    int ld;
    __device__ half8 high(int r, int p) const { return *reinterpret_cast<const half8 *>(h + piece_at(r, p, ld)); }
    __device__ half8 low(int r, int p) const { return *reinterpret_cast<const half8 *>(l + piece_at(r, p, ld)); }
    __device__ int at(int r, int c) const { return piece_at(r, c / 8, ld) + c % 8; }
};

// acc += P Q^T over the kSpan values from k0 of 32 rows from pr and 32 from qr
template <int kSpan>
__device__ inline float16v block_product(const Planes &P, int pr, const Planes &Q, int qr, int k0, float16v acc)
{
    const int lane = lane_id(), r = lane % 32;
    float16v mixed = {};
#pragma unroll
    for (int kk = 0; kk < kSpan / 16; ++kk) {
        const int k = k0 / 8 + 2 * kk + lane / 32;
        const half8 ph = P.high(pr + r, k), pl = P.low(pr + r, k), qh = Q.high(qr + r, k), ql = Q.low(qr + r, k);
        mixed = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, mixed, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
        mixed = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, mixed, 0, 0, 0);
    }
    return acc + mixed;
}

// row of accumulator value 4 q, of which the next three follow (columns: lane % 32)
__device__ inline int acc_row(int q) { return 8 * q + 4 * (lane_id() / 32); }

// four values of an accumulator as halves
__device__ inline void split4(const float *v, half4 &h, half4 &l)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        f16 vh, vl;
        split(v[r], vh, vl);
        h[r] = vh;
        l[r] = vl;
    }
}

// kAll: one block a matrix, every step.  Otherwise launch `k`: 0 loads U's slice and leaves its Gram matrix, k > 0
// makes step k - 1.  summed: the Gram matrices have been added up.
template <typename E, int MB, bool kAll>
__global__ __launch_bounds__(kNarrowBlock) void orth_narrow_kernel(OrthArgs a, char *ws, NarrowLayout L, int k, int summed)
{
    constexpr int kM = 32 * MB;
    constexpr int kGroups = kAll ? int(kNarrowWhole / kM / 64) : kSlice / 64; // 64 columns each, W / 64 of them in use
    constexpr int kPer = kM * 64 / kNarrowBlock;                             // values of a group and thread
    extern __shared__ __align__(16) char s_mem[];
    __shared__ double s_norm[kNarrowBlock / kWave];
    const int W = L.width;
    f16 *mem = reinterpret_cast<f16 *>(s_mem);
    const Planes X = {mem, mem + kM * W, W};
    const Planes T = {mem + 2 * kM * W, mem + 3 * kM * W, kM};
    const Planes A = {mem + 4 * kM * W, mem + 4 * kM * W + kM * kM, kM};
    float4 *scratch = reinterpret_cast<float4 *>(A.h); // partial products, before A's planes take the place
    const int tid = threadIdx.x, lane = lane_id(), w = tid / kWave;
    const bool wide = a.rows <= a.cols;
    const int m = int(wide ? a.rows : a.cols);
    const int64_t n = wide ? a.cols : a.rows;
    const int64_t z = blockIdx.y, j0 = int64_t(blockIdx.x) * W;
    char *base = ws + z * L.stride;
    const int64_t g_i = wide ? a.g_stride : 1, g_j = wide ? 1 : a.g_stride; // steps along m and along n
    const int64_t m_i = wide ? a.m_stride : 1, m_j = wide ? 1 : a.m_stride;
    const int64_t w_i = wide ? a.w_stride : 1, w_j = wide ? 1 : a.w_stride;
    const int cols = int(n - j0 < W ? n - j0 : W);

    if (kAll || k == 0) {
        // U in registers, between one read and the scaled planes
        float u[kGroups * kPer];
        // value q of group g is at (ti + q di, tj + q dj + 64 g): along the rows of the caller's matrix
        const int ti = wide ? tid / 64 : tid % kM, tj = wide ? tid % 64 : tid / kM;
        const int di = wide ? kNarrowBlock / 64 : 0, dj = wide ? 0 : kNarrowBlock / kM;
        const auto place = [&](int g, int q, int &i, int &j) {
            i = ti + q * di;
            j = tj + q * dj + 64 * g;
        };
        const E *G = static_cast<const E *>(a.G) + z * a.g_batch + j0 * g_j + (ti * g_i + tj * g_j);
        float *M = a.M ? a.M + z * a.m_batch + j0 * m_j + (ti * m_i + tj * m_j) : nullptr;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                int i, j;
                place(g, q, i, j);
                u[g * kPer + q] = i < m && j < cols ? float(G[q * (di * g_i + dj * g_j) + g * (64 * g_j)]) : 0.0f;
            }
        if (M) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                float mo[kPer];
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    int i, j;
                    place(g, q, i, j);
                    mo[q] = i < m && j < cols ? M[q * (di * m_i + dj * m_j) + g * (64 * m_j)] : 0.0f;
                }
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    int i, j;
                    place(g, q, i, j);
                    if constexpr (kAll) {
                        mo[q] = a.momentum * mo[q] + u[g * kPer + q];
                        if (i < m && j < cols) M[q * (di * m_i + dj * m_j) + g * (64 * m_j)] = mo[q];
                    } // else a launch before has done so
                    u[g * kPer + q] = update_value(a, u[g * kPer + q], mo[q]);
                }
            }
        }
        // the norm: of this block's values, or of the partial sums that a launch before left
        double sum = 0.0;
        if constexpr (kAll) {
#pragma unroll
            for (int q = 0; q < kGroups * kPer; ++q) sum += double(u[q]) * double(u[q]);
        } else {
            const double *part = reinterpret_cast<const double *>(base + L.norm);
            if (tid < L.norm_blocks) sum = part[tid]; // kOrthNormBlocks at most
        }
        sum = wave_sum(sum);
        if (lane == 0) s_norm[w] = sum;
        __syncthreads();
        sum = 0.0;
        for (int v = 0; v < kNarrowBlock / kWave; ++v) sum += s_norm[v];
        const double scale = double(a.step[0].sx) / (sqrt(sum) + a.eps);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g * 64 >= W) break;
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                int i, j;
                place(g, q, i, j);
                f16 h, l;
                split(float(double(u[g * kPer + q]) * scale), h, l);
                X.h[X.at(i, j)] = T.h[T.at(j, i)] = h;
                X.l[X.at(i, j)] = T.l[T.at(j, i)] = l;
            }
        }
    } else {
        const half8 *planes = reinterpret_cast<const half8 *>(base + L.x) + j0 * (kM / 8);
#pragma unroll
        for (int q = 0; q < kSlice * (kM / 8) / kNarrowBlock; ++q) {
            const int e = tid + q * kNarrowBlock, j = e / (kM / 8), p = e % (kM / 8);
            *reinterpret_cast<half8 *>(T.h + piece_at(j, p, kM)) = planes[e];
            *reinterpret_cast<half8 *>(T.l + piece_at(j, p, kM)) = planes[L.n * (kM / 8) + e];
        }
    }
    __syncthreads();

    const int first = kAll ? 0 : (k == 0 ? 0 : k - 1), last = kAll ? a.steps : (k == 0 ? 0 : k);
    constexpr int kBlocks = MB * MB;             // 32 x 32 blocks of A
    constexpr int kParts = MB == 1 ? 4 : 2;      // waves that share one block's sum
    const int ib = (w % kBlocks) / MB * 32, jb = (w % kBlocks) % MB * 32, part = w / kBlocks;
    const bool worker = part < kParts;

    // the Gram matrix of X as it is in LDS, the block (ib, jb) in waves below kBlocks
    const auto gram = [&]() {
        float16v acc = {};
        if (worker)
            for (int k0 = part * 32; k0 < W; k0 += kParts * 32) acc = block_product<32>(X, ib, X, jb, k0, acc);
        if (worker && part > 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                scratch[(((part - 1) * kBlocks + w % kBlocks) * 4 + q) * kWave + lane] =
                    make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
        }
        __syncthreads();
        if (w < kBlocks) {
#pragma unroll
            for (int p = 0; p + 1 < kParts; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 v = scratch[((p * kBlocks + w) * 4 + q) * kWave + lane];
                    acc[4 * q] += v.x;
                    acc[4 * q + 1] += v.y;
                    acc[4 * q + 2] += v.z;
                    acc[4 * q + 3] += v.w;
                }
        }
        __syncthreads();
        return acc;
    };
    // partial Gram matrices keep the accumulators' own order: [block][4][64 lanes][4]
    const auto partials = [&](int which) { return reinterpret_cast<float4 *>(base + L.gram[which & 1]); };

    for (int s = first; s < last; ++s) {
        const OrthStep &S = a.step[s];
        const float to_a = S.sa / (S.sx * S.sx);
        // A, then B in its place.  Both are symmetric: the value at (row, column) is stored at (column, row),
        // where four rows of an accumulator lie side by side
        const int c = jb + lane % 32;
        if constexpr (kAll) {
            const float16v acc = gram();
            if (w < kBlocks) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = acc[4 * q + r] * to_a;
                    half4 h, l;
                    split4(v, h, l);
                    *reinterpret_cast<half4 *>(A.h + A.at(c, ib + acc_row(q))) = h;
                    *reinterpret_cast<half4 *>(A.l + A.at(c, ib + acc_row(q))) = l;
                }
            }
        } else {
            // every thread adds up four values at a time over the slices
            const float4 *src = summed ? reinterpret_cast<const float4 *>(base + L.total) : partials(k - 1);
            const int count = summed ? 1 : L.slices;
            for (int e = tid; e < kM * kM / 4; e += kNarrowBlock) {
                float v[4] = {};
#pragma unroll 8
                for (int q = 0; q < count; ++q) {
                    const float4 x = src[q * (kM * kM / 4) + e];
                    v[0] += x.x;
                    v[1] += x.y;
                    v[2] += x.z;
                    v[3] += x.w;
                }
                const int b = e / 256, q = e / 64 % 4, ln = e % 64;
                const int row = (b % MB) * 32 + ln % 32, col = (b / MB) * 32 + 8 * q + 4 * (ln / 32);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] *= to_a;
                half4 h, l;
                split4(v, h, l);
                *reinterpret_cast<half4 *>(A.h + A.at(row, col)) = h;
                *reinterpret_cast<half4 *>(A.l + A.at(row, col)) = l;
            }
        }
        __syncthreads();
        half4 bh[4], bl[4];
        if (w < kBlocks) {
            const float16v sq = block_product<kM>(A, ib, A, jb, 0, float16v{});
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const half4 h = *reinterpret_cast<const half4 *>(A.h + A.at(c, ib + acc_row(q)));
                const half4 l = *reinterpret_cast<const half4 *>(A.l + A.at(c, ib + acc_row(q)));
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    v[r] = (float(h[r]) + float(l[r])) * (S.b * S.sb / S.sa) + sq[4 * q + r] * (S.c * S.sb / (S.sa * S.sa));
                    if (ib + acc_row(q) + r == c) v[r] += S.a * S.sb;
                }
                split4(v, bh[q], bl[q]);
            }
        }
        __syncthreads();
        if (w < kBlocks) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                *reinterpret_cast<half4 *>(A.h + A.at(c, ib + acc_row(q))) = bh[q];
                *reinterpret_cast<half4 *>(A.l + A.at(c, ib + acc_row(q))) = bl[q];
            }
        }
        __syncthreads();
        // X <- B X in 32 x 32 blocks, two a wave at most; in place, once every wave has read its columns
        const bool done = s + 1 == a.steps;
        const float xs = (done ? 1.0f : a.step[s + 1].sx) / (S.sb * S.sx);
        const int items = W / 32 * MB;
        float16v x[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int item = w + t * (kNarrowBlock / kWave);
            if (item < items) x[t] = block_product<kM>(A, item % MB * 32, T, item / MB * 32, 0, float16v{});
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int item = w + t * (kNarrowBlock / kWave);
            if (item >= items) continue;
            const int i0 = item % MB * 32, j = item / MB * 32 + lane % 32;
            if (done) {
                E *out = static_cast<E *>(a.W) + z * a.w_batch + (j0 + j) * w_j;
                float old[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = i0 + acc_row(r / 4) + r % 4;
                    old[r] = a.M && i < m && j < cols ? float(out[i * w_i]) : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = i0 + acc_row(r / 4) + r % 4;
                    const float v = x[t][r] * xs;
                    if (i < m && j < cols) out[i * w_i] = E(a.M ? a.keep * old[r] - a.rate * v : v);
                }
                continue;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = i0 + acc_row(q);
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = x[t][4 * q + r] * xs;
                half4 h, l;
                split4(v, h, l);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    X.h[X.at(i + r, j)] = h[r];
                    X.l[X.at(i + r, j)] = l[r];
                }
                *reinterpret_cast<half4 *>(T.h + T.at(j, i)) = h;
                *reinterpret_cast<half4 *>(T.l + T.at(j, i)) = l;
            }
        }
        __syncthreads();
    }
    if (kAll || k == a.steps) return;
    const float16v acc = gram();
    if (w < kBlocks) {
        float4 *dst = partials(k) + int64_t(blockIdx.x) * (kM * kM / 4) + w * 4 * kWave + lane;
#pragma unroll
        for (int q = 0; q < 4; ++q) dst[q * kWave] = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    }
    half8 *planes = reinterpret_cast<half8 *>(base + L.x) + j0 * (kM / 8);
#pragma unroll
    for (int q = 0; q < kSlice * (kM / 8) / kNarrowBlock; ++q) {
        const int e = tid + q * kNarrowBlock, j = e / (kM / 8), p = e % (kM / 8);
        planes[e] = *reinterpret_cast<const half8 *>(T.h + piece_at(j, p, kM));
        planes[L.n * (kM / 8) + e] = *reinterpret_cast<const half8 *>(T.l + piece_at(j, p, kM));
    }
}

// adds up the slices' Gram matrices: a block takes 64 of its values and four strands of slices
__global__ __launch_bounds__(256) void orth_sum_kernel(char *ws, NarrowLayout L, int which, int values)
{
    __shared__ float s_sum[4][kWave];
    char *base = ws + int64_t(blockIdx.y) * L.stride;
    const int v = int(blockIdx.x) * kWave + threadIdx.x % kWave, strand = threadIdx.x / kWave;
    const float *src = reinterpret_cast<const float *>(base + L.gram[which & 1]);
    float s = 0.0f;
#pragma unroll 8
    for (int q = strand; q < L.slices; q += 4) s += src[int64_t(q) * values + v];
    s_sum[strand][threadIdx.x % kWave] = s;
    __syncthreads();
    if (strand == 0)
        reinterpret_cast<float *>(base + L.total)[v] = (s_sum[0][v % kWave] + s_sum[1][v % kWave]) + (s_sum[2][v % kWave] + s_sum[3][v % kWave]);
}

template <typename E, int MB> void run_narrow(const OrthArgs &a, char *ws, const NarrowLayout &L, hipStream_t st)
{
    constexpr int kM = 32 * MB;
    const size_t lds = size_t(kM) * L.width * 8 + (MB == 1 ? 3 * 4096 : 4 * 4096);
    const dim3 grid(uint32_t(L.slices), uint32_t(a.batch));
    if (L.slices == 1) {
        orth_narrow_kernel<E, MB, true><<<grid, kNarrowBlock, lds, st>>>(a, ws, L, 0, 0);
        return;
    }
    orth_norm_kernel<<<dim3(L.norm_blocks, uint32_t(a.batch)), 256, 0, st>>>(a, ws, int64_t(L.stride), L.norm);
    const bool sum = L.slices > kSliceSum;
    for (int k = 0; k <= a.steps; ++k) {
        if (k > 0 && sum) orth_sum_kernel<<<dim3(kM * kM / kWave, uint32_t(a.batch)), 256, 0, st>>>(ws, L, k - 1, kM * kM);
        orth_narrow_kernel<E, MB, false><<<grid, kNarrowBlock, lds, st>>>(a, ws, L, k, sum);
    }
}
template <typename E> void run_narrow_type(const OrthArgs &a, char *ws, const NarrowLayout &L, hipStream_t st)
{
    if (L.blocks == 1)
        run_narrow<E, 1>(a, ws, L, st);
    else
        run_narrow<E, 2>(a, ws, L, st);
}

} // namespace

int norm_blocks_of(int64_t rows, int64_t cols)
{
    const int64_t want = (rows * cols + 4095) / 4096;
    return int(want < kOrthNormBlocks ? want : kOrthNormBlocks);
}

NarrowLayout make_narrow_layout(int64_t rows, int64_t cols)
{
    NarrowLayout L;
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    L.blocks = m <= 32 ? 1 : 2;
    const int64_t side = 32 * L.blocks, whole = (n + 63) / 64 * 64;
    // one launch as long as X fits LDS: 8 bytes a value
    L.width = int(whole * side <= kNarrowWhole ? whole : kSlice);
    L.slices = int((n + L.width - 1) / L.width);
    L.n = int64_t(L.slices) * L.width;
    L.norm_blocks = norm_blocks_of(rows, cols);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    L.x = take(2 * sizeof(f16) * size_t(L.n * side));
    for (int k = 0; k < 2; ++k) L.gram[k] = take(sizeof(float) * size_t(side * side) * size_t(L.slices));
    L.total = take(sizeof(float) * size_t(side * side));
    L.norm = take(sizeof(double) * kOrthNormBlocks);
    L.stride = at;
    return L;
}

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

size_t orth_workspace(int64_t rows, int64_t cols)
{
    return orth_narrow(rows, cols) ? make_narrow_layout(rows, cols).stride : make_orth_layout(rows, cols).stride;
}

void launch_orthogonalise(const OrthArgs &a, void *workspace, hipStream_t st)
{
    if (a.batch == 0) return;
    char *ws = static_cast<char *>(workspace);
    if (orth_narrow(a.rows, a.cols)) {
        const NarrowLayout L = make_narrow_layout(a.rows, a.cols);
        if (a.type == Elem::kF32)
            run_narrow_type<float>(a, ws, L, st);
        else if (a.type == Elem::kF16)
            run_narrow_type<f16>(a, ws, L, st);
        else
            run_narrow_type<bf16>(a, ws, L, st);
        return;
    }
    const OrthLayout L = make_orth_layout(a.rows, a.cols);
    const int norm_blocks = norm_blocks_of(a.rows, a.cols);
    orth_norm_kernel<<<dim3(norm_blocks, uint32_t(a.batch)), 256, 0, st>>>(a, ws, int64_t(L.stride), L.norm);
    orth_planes_kernel<<<dim3(uint32_t(L.cols / kT), uint32_t(L.rows / kT), uint32_t(a.batch)), 256, 0, st>>>(a, ws, L, norm_blocks);
    if (a.type != Elem::kBF16)
        run_steps<true>(a, ws, L, st);
    else
        run_steps<false>(a, ws, L, st);
}

} // namespace bht
