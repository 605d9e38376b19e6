// The product C = A B^T of row-major operands on the matrix cores, with an
// epilogue of the caller's: A's rows are points, B's rows are features.
//
// All types go through one loop on bytes.  A block makes a tile of kM points x
// kN rows of B; slices of 128 bytes of every row (32 fp32, 64 fp16 or bf16, 128
// int8 values) go through a ring in LDS.  A row's eight 16-byte pieces are stored
// in an order that depends on the row (piece c of row r in place c ^ (r % 8)), so
// that the lanes of a fragment read, which take the same piece of 16 rows, fall on
// different banks.  A fragment is 16 bytes a lane: row lane % 16, piece lane / 16
// of a half slice, which is what one matrix instruction takes of 16 and 8 bits;
// fp32 takes four, each with one of a piece's values (the sum over K has the same
// terms in another order).
//
// Features are the columns of the instruction's output and points its rows, so a
// lane holds 4 points of a feature a block; B's rows are put into LDS in an order
// that makes the lane's blocks consecutive features.  Outputs go to memory from
// registers: a lane stores its features of a point as one vector, and 16 lanes
// next to each other a run of the point's (64 bytes or more of tiles of 128 on).
// Lanes side by side have to be neighbours in memory for that: with points along
// the lanes, each lane's 16 bytes were a request of its own.
#pragma once

#include <type_traits>

#include "dense.hpp"

namespace bht {
namespace prod {

typedef int32_t int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef bf16 bhalf8 __attribute__((ext_vector_type(8)));

typedef int4v Piece; // 16 bytes of a row
constexpr int kSlice = 128;

template <typename E> struct Ops;
template <> struct Ops<f16> {
    typedef float4v Acc;
    static __device__ inline Acc mul(Piece p, Piece q, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, p), __builtin_bit_cast(half8, q), c, 0, 0, 0);
    }
};
template <> struct Ops<bf16> {
    typedef float4v Acc;
    static __device__ inline Acc mul(Piece p, Piece q, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, p), __builtin_bit_cast(bhalf8, q), c, 0, 0, 0);
    }
};
template <> struct Ops<int8_t> {
    typedef int4v Acc;
    static __device__ inline Acc mul(Piece p, Piece q, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(p, q, c, 0, 0, 0); }
};
template <> struct Ops<float> {
    typedef float4v Acc;
    static __device__ inline Acc mul(Piece p, Piece q, Acc c)
    {
        const float4v a = __builtin_bit_cast(float4v, p), b = __builtin_bit_cast(float4v, q);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

template <int M, int N, int Wm, int Wn, int Stages> struct Tile {
    static constexpr int kM = M, kN = N, kWm = Wm, kWn = Wn, kStages = Stages;
    static constexpr int kWaves = Wm * Wn, kThreads = kWaves * kWave;
    static constexpr int kI = M / Wm / 16, kJ = N / Wn / 16; // 16 x 16 blocks of a wave: points, rows of B
    static constexpr int kGroups = (M + N) / 8;              // groups of 8 rows in a slice, A's first
    static constexpr int kEach = kGroups / kWaves;           // groups a wave loads
    static constexpr int kBuffer = (M + N) * kSlice;         // bytes
    static_assert(kGroups % kWaves == 0 && M % (16 * Wm) == 0 && N % (16 * Wn) == 0, "even shares");
};

typedef Tile<256, 256, 2, 4, 2> TileLarge;
typedef Tile<128, 128, 2, 2, 2> TileMiddle;
typedef Tile<64, 64, 2, 2, 3> TileSmall;

// How a product's operands lie.  kRows: C = A B^T of rows as above.  kDual: two such products of one A, by B and B2, whose
// values a lane has side by side.  kColumns: C = A^T B, both summed over their rows (points): a slice is so many rows that
// its columns are kSlice bytes high, and fragments are read across the rows (16-bit values by transposing LDS loads).
enum class Form { kRows, kDual, kColumns };

// Operands and grid of a product.
struct Product {
    const char *A, *B, *B2;
    int64_t a_stride, b_stride, b2_stride; // bytes between rows
    int64_t rows, features;                // of the output (kColumns: columns of A and of B)
    int64_t bytes;                         // of a row; kColumns: rows summed over, times the size of a value
    int32_t down, across;        // tiles
    int32_t slices, per_split;   // of a row, and of a split (blockIdx.y)
};

__device__ __align__(16) const char kZeros[16] = {};

// Where the b-th tile lies: blocks are dealt to the 8 XCDs in turn and each XCD gets consecutive tiles, four rows of
// tiles at a time, column by column.
__device__ inline void place(const Product &a, uint32_t b, int32_t &bi, int32_t &bj)
{
    const uint32_t tiles = uint32_t(a.down) * uint32_t(a.across);
    const uint32_t x = b % 8, q = tiles / 8, r = tiles % 8;
    const uint32_t t = x * q + (x < r ? x : r) + b / 8;
    const uint32_t group = t / (4u * uint32_t(a.across)), in = t - group * 4u * uint32_t(a.across), top = group * 4;
    const uint32_t left = uint32_t(a.down) - top, high = left < 4 ? left : 4;
    bj = int32_t(in / high);
    bi = int32_t(top + in % high);
}

// 16 bytes of a row at p, of elements at their own alignment, with `left` bytes from p to the row's end: zeros behind it.
// The last piece is the row's last 16 bytes, shifted; a row that has fewer is read value by value.
template <typename E> __device__ inline Piece any_piece(const char *row, int64_t at, int64_t bytes)
{
    if (bytes < 16) { // the same for all lanes
        constexpr int kV = 16 / int(sizeof(E));
        E x[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            const bool there = at + e * int(sizeof(E)) < bytes;
            const E v = *reinterpret_cast<const E *>(row + (there ? at + e * int(sizeof(E)) : 0));
            x[e] = there ? v : E(0);
        }
        Piece v;
        __builtin_memcpy(&v, x, 16);
        return v;
    }
    const int64_t most = bytes - 16;
    const int over = int(at <= most ? 0 : at - most < 16 ? at - most : 16); // bytes behind the end
    uint64_t v[2];
    __builtin_memcpy(v, row + (over == 0 ? at : most), 16);
    const int s = 8 * over;
    const uint64_t low = s == 0 ? v[0] : s < 64 ? v[0] >> s | v[1] << (64 - s) : s < 128 ? v[1] >> (s - 64) : 0;
    const uint64_t high = s < 64 ? v[1] >> s : 0;
    const uint64_t both[2] = {low, high};
    Piece r;
    __builtin_memcpy(&r, both, 16);
    return r;
}
// ... of a piece that lies inside its row
__device__ inline Piece inner_piece(const char *p)
{
    Piece v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// Columns in LDS: `kPitch` bytes a row.  The blocks of 16 columns of a row are stored in an order that depends on the row, such
// that what 32 lanes take of a block (16 bits: rows 0 to 3 and 8 to 11 of it; 32 bits: four rows) falls on different banks.
template <typename E, int kPitch> __device__ inline int column_turn(int row)
{
    if (sizeof(E) == 4) return row & 3;
    return kPitch < 256 ? (row >> 1 & 1) | (row >> 3 & 1) << 1 : (row & 3) | (row >> 3 & 1) << 2;
}
// Piece c of a row's, and the place it is stored in, either way
template <typename E, int kPitch> __device__ inline int column_piece(int c, int row) { return c ^ (int(sizeof(E)) * column_turn<E, kPitch>(row)); }

// What a lane takes of columns 16 `block` .. in half a slice: a fragment's values for column lane % 16.  16 bits: a transposing
// load gives 4 x 16 values of each 16 lanes, which name the four rows' pieces; two make the 8 rows of a lane.  32 bits: one by one.
// column_place: the lane's part of the address (rows further down turn alike).
template <typename E, int kPitch> __device__ inline int column_place(int block)
{
    const int lane = lane_id(), row = sizeof(E) == 2 ? lane / 16 * 8 + lane % 16 / 4 : lane / 16;
    return row * kPitch + (block ^ column_turn<E, kPitch>(row)) * (16 * int(sizeof(E))) + (sizeof(E) == 2 ? lane % 4 * 8 : lane % 16 * 4);
}
// N of them (2 or 4), kOffset bytes behind `at`.  The transposing loads are written out, with their wait: before the builtin
// the compiler waits for every load into LDS that is under way, whatever it fills (16384 x 512 to 2048 108 us, 2.3 a slice).
template <typename E, int kPitch, int kOffset, int N> __device__ inline void column_fragments(const char *const (&at)[N], Piece (&v)[N])
{
    static_assert(N == 2 || N == 4, "written out for these");
    if constexpr (sizeof(E) == 2) {
        typedef int32_t Two __attribute__((ext_vector_type(2)));
        typedef const __attribute__((address_space(3))) char *Place;
        Two low[N], high[N];
        if constexpr (N == 4) {
            asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                         "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
                         "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
                         "ds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %6, %11 offset:%12\n\t"
                         "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(low[0]), "=&v"(high[0]), "=&v"(low[1]), "=&v"(high[1]), "=&v"(low[2]), "=&v"(high[2]), "=&v"(low[3]), "=&v"(high[3])
                         : "v"((Place)at[0]), "v"((Place)at[1]), "v"((Place)at[2]), "v"((Place)at[3]), "n"(kOffset), "n"(kOffset + 4 * kPitch)
                         : "memory");
        } else {
            asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\t"
                         "ds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                         "ds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                         "ds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(low[0]), "=&v"(high[0]), "=&v"(low[1]), "=&v"(high[1])
                         : "v"((Place)at[0]), "v"((Place)at[1]), "n"(kOffset), "n"(kOffset + 4 * kPitch)
                         : "memory");
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = Piece{low[i][0], low[i][1], high[i][0], high[i][1]};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = *reinterpret_cast<const int32_t *>(at[i] + kOffset + 4 * e * kPitch);
    }
}
// ... and both halves of a slice, with one wait
template <typename E, int kPitch, int kOffset, int N> __device__ inline void column_slices(const char *const (&at)[N], Piece (&v)[2][N])
{
    static_assert(N == 2 || N == 4, "written out for these");
    constexpr int kHalf = (sizeof(E) == 2 ? 32 : 16) * kPitch;
    if constexpr (sizeof(E) == 2 && N == 4) {
        typedef int32_t Two __attribute__((ext_vector_type(2)));
        typedef const __attribute__((address_space(3))) char *Place;
        Two x[16];
        asm volatile("ds_read_b64_tr_b16 %0, %16 offset:%20\n\t"
                     "ds_read_b64_tr_b16 %1, %16 offset:%21\n\t"
                     "ds_read_b64_tr_b16 %2, %17 offset:%20\n\t"
                     "ds_read_b64_tr_b16 %3, %17 offset:%21\n\t"
                     "ds_read_b64_tr_b16 %4, %18 offset:%20\n\t"
                     "ds_read_b64_tr_b16 %5, %18 offset:%21\n\t"
                     "ds_read_b64_tr_b16 %6, %19 offset:%20\n\t"
                     "ds_read_b64_tr_b16 %7, %19 offset:%21\n\t"
                     "ds_read_b64_tr_b16 %8, %16 offset:%22\n\t"
                     "ds_read_b64_tr_b16 %9, %16 offset:%23\n\t"
                     "ds_read_b64_tr_b16 %10, %17 offset:%22\n\t"
                     "ds_read_b64_tr_b16 %11, %17 offset:%23\n\t"
                     "ds_read_b64_tr_b16 %12, %18 offset:%22\n\t"
                     "ds_read_b64_tr_b16 %13, %18 offset:%23\n\t"
                     "ds_read_b64_tr_b16 %14, %19 offset:%22\n\t"
                     "ds_read_b64_tr_b16 %15, %19 offset:%23\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]),
                       "=&v"(x[9]), "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
                     : "v"((Place)at[0]), "v"((Place)at[1]), "v"((Place)at[2]), "v"((Place)at[3]), "n"(kOffset), "n"(kOffset + 4 * kPitch),
                       "n"(kOffset + kHalf), "n"(kOffset + kHalf + 4 * kPitch)
                     : "memory");
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[h][i] = Piece{x[8 * h + 2 * i][0], x[8 * h + 2 * i][1], x[8 * h + 2 * i + 1][0], x[8 * h + 2 * i + 1][1]};
    } else if constexpr (sizeof(E) == 2) {
        const char *const four[4] = {at[0], at[1], at[0] + kHalf, at[1] + kHalf};
        Piece x[4];
        column_fragments<E, kPitch, kOffset>(four, x);
        v[0][0] = x[0];
        v[0][1] = x[1];
        v[1][0] = x[2];
        v[1][1] = x[3];
    } else {
        column_fragments<E, kPitch, kOffset>(at, v[0]);
        column_fragments<E, kPitch, kOffset + kHalf>(at, v[1]);
    }
}

// A wave's blocks: acc[i][j] holds points 16 i .. against rows 16 j .. of the wave's part of B.  kDual: the first half of
// the blocks j is B's, the second B2's.  kAny: rows of any alignment and length, through registers; else rows, their
// strides and lengths are multiples of 16 bytes and loads write LDS directly.
template <typename E, typename T, Form kForm, bool kAny>
__device__ inline void multiply_tile(const Product &a, int32_t bi, int32_t bj, typename Ops<E>::Acc (&acc)[T::kI][T::kJ])
{
    extern __shared__ __align__(16) char s_mem[];
    constexpr bool kDual = kForm == Form::kDual, kColumns = kForm == Form::kColumns;
    constexpr int kEs = int(sizeof(E)), kTogether = kDual ? T::kJ / 2 : T::kJ; // blocks whose rows are a lane's consecutive features
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();
    const int32_t first = int32_t(blockIdx.y) * a.per_split;
    const int32_t slices = (first + a.per_split < a.slices ? first + a.per_split : a.slices) - first;

    // this lane's piece of each kilobyte that the wave loads, and where that ends: bytes left of the row (of the column)
    const char *src[T::kEach];
    int64_t left[kColumns ? T::kEach : 1], step[2]; // step: from slice to slice, of A and of B
    left[0] = a.bytes - int64_t(first) * kSlice - ((lane % 8) ^ (lane / 8)) * 16;
    step[0] = kColumns ? kSlice / kEs * a.a_stride : kSlice;
    step[1] = kColumns ? kSlice / kEs * a.b_stride : kSlice;
#pragma unroll
    for (int e = 0; e < T::kEach; ++e) {
        const bool in_a = (e * T::kWaves + w) * 8 < T::kM;
        if constexpr (kColumns) {
            const int part = (e * T::kWaves + w) * 8 - (in_a ? 0 : T::kM); // eighths of a kilobyte before this one
            const int pieces = (in_a ? T::kM : T::kN) * kEs / 16, at = part * 8 + lane, row = at / pieces;
            const int turned = in_a ? column_piece<E, T::kM * kEs>(at % pieces, row) : column_piece<E, T::kN * kEs>(at % pieces, row);
            const int64_t column = int64_t(in_a ? bi * T::kM : bj * T::kN) * kEs + turned * 16;
            const int64_t most = (in_a ? a.rows : a.features) * kEs - 16, stride = in_a ? a.a_stride : a.b_stride;
            src[e] = (in_a ? a.A : a.B) + (int64_t(first) * (kSlice / kEs) + row) * stride + (column < most ? column : most);
            left[e] = a.bytes - int64_t(first) * kSlice - row * kEs;
        } else {
            const int row = (e * T::kWaves + w) * 8 + lane / 8;
            if (in_a) {
                const int64_t at = int64_t(bi) * T::kM + row;
                src[e] = a.A + (at < a.rows ? at : a.rows - 1) * a.a_stride;
            } else {
                const int in = row - T::kM, part = in % (16 * T::kJ), block = part / 16, i = part % 16;
                const bool second = kDual && block >= kTogether;
                const int64_t at = int64_t(bj) * (kDual ? T::kN / 2 : T::kN) + in / (16 * T::kJ) * (16 * kTogether) + i * kTogether
                                   + (second ? block - kTogether : block);
                const int64_t held = at < a.features ? at : a.features - 1;
                src[e] = second ? a.B2 + held * a.b2_stride : a.B + held * a.b_stride;
            }
            if constexpr (!kAny) src[e] += int64_t(first) * kSlice + ((lane % 8) ^ (lane / 8)) * 16;
        }
    }
    const int wi = w / T::kWn * (T::kI * 16), wj = w % T::kWn * (T::kJ * 16);
    const auto fragment = [&](const char *in, int row, int piece) {
        return *reinterpret_cast<const Piece *>(in + row * kSlice + ((piece ^ (row & 7)) * 16));
    };
    Piece p[2][T::kI], q[2][T::kJ];
    int own_a[T::kI], own_b[T::kJ]; // kColumns: the lane's places
    if constexpr (kColumns) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i) own_a[i] = column_place<E, T::kM * kEs>(wi / 16 + i);
#pragma unroll
        for (int j = 0; j < T::kJ; ++j) own_b[j] = T::kM * kSlice + column_place<E, T::kN * kEs>(wj / 16 + j);
    }
    const auto read = [&](const char *in, int half) {
        if constexpr (kColumns) {
            const char *a_at[T::kI], *b_at[T::kJ];
            constexpr int kRows = kSlice / kEs / 2;
#pragma unroll
            for (int i = 0; i < T::kI; ++i) a_at[i] = in + own_a[i] + half * kRows * T::kM * kEs;
#pragma unroll
            for (int j = 0; j < T::kJ; ++j) b_at[j] = in + own_b[j] + half * kRows * T::kN * kEs;
            column_fragments<E, T::kN * kEs, 0>(b_at, q[half]);
            column_fragments<E, T::kM * kEs, 0>(a_at, p[half]);
            return;
        }
        const int piece = half * 4 + lane / 16;
#pragma unroll
        for (int j = 0; j < T::kJ; ++j) q[half][j] = fragment(in, T::kM + wj + 16 * j + lane % 16, piece);
#pragma unroll
        for (int i = 0; i < T::kI; ++i) p[half][i] = fragment(in, wi + 16 * i + lane % 16, piece);
    };
    const auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < T::kI; ++i)
#pragma unroll
            for (int j = 0; j < T::kJ; ++j) acc[i][j] = Ops<E>::mul(p[half][i], q[half][j], acc[i][j]);
    };

    if constexpr (kAny) {
        Piece x[T::kEach];
        const auto load = [&](int slice) {
            const int64_t at = int64_t(first + slice) * kSlice + ((lane % 8) ^ (lane / 8)) * 16;
            if (int64_t(first + slice + 1) * kSlice <= a.bytes) {
#pragma unroll
                for (int e = 0; e < T::kEach; ++e) x[e] = inner_piece(src[e] + at);
            } else {
#pragma unroll
                for (int e = 0; e < T::kEach; ++e) x[e] = any_piece<E>(src[e], at, a.bytes);
            }
        };
        load(0);
        for (int slice = 0; slice < slices; ++slice) {
            char *to = s_mem + slice % 2 * T::kBuffer;
#pragma unroll
            for (int e = 0; e < T::kEach; ++e)
                *reinterpret_cast<Piece *>(to + (e * T::kWaves + w) * 8 * kSlice + lane * 16) = x[e];
            __syncthreads(); // the other buffer's readers are past it too: they have written this one
            if (slice + 1 < slices) load(slice + 1);
            read(to, 0);
            read(to, 1);
            multiply(0);
            multiply(1);
        }
    } else {
        constexpr int kLoads = T::kEach;
        const auto fetch = [&](int slice) {
            // past the end the last slice again, into a buffer that nobody reads: every wait counts alike
            const int32_t k = slice < slices ? slice : slices - 1;
            char *to = s_mem + slice % T::kStages * T::kBuffer;
#pragma unroll
            for (int e = 0; e < T::kEach; ++e) {
                const bool zero = left[kColumns ? e : 0] - int64_t(k) * kSlice <= 0; // behind the end
                const char *from = zero ? kZeros : src[e] + k * step[(e * T::kWaves + w) * 8 < T::kM ? 0 : 1];
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                                 (__attribute__((address_space(3))) void *)(to + (e * T::kWaves + w) * 8 * kSlice),
                                                 16, 0, 0);
            }
        };
#pragma unroll
        for (int e = 0; e < T::kStages; ++e) fetch(e);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((T::kStages - 1) * kLoads) : "memory");
        read(s_mem, 0);
        for (int slice = 0; slice < slices; ++slice) {
            read(s_mem + slice % T::kStages * T::kBuffer, 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            // this wave's loads of the next slice have landed and its reads of this one are done; then everybody's
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((T::kStages - 2) * kLoads) : "memory");
            fetch(slice + T::kStages);
            read(s_mem + (slice + 1) % T::kStages * T::kBuffer, 0); // behind the last slice: not used
            __builtin_amdgcn_sched_barrier(0);
            multiply(1);
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); // no load is under way when the block's LDS is given on
    }
}

// ------------------------------------------------------------------ few points
// A block makes 16 features of 16 kI points, its waves share K out in slices, every kFewWaves-th each, and take fragments
// straight from memory: the weights are read once for so many points, a line of 16 rows at a time.  Rows of any alignment.
// For up to 16 points; and for more where tiles are so few that each one's slices, one after another, are what takes time.
// x(slice, half, i): the points' fragment, zeros behind the end.  ready(): called once by every wave while the first weights
// are under way.
constexpr int kFewWaves = 8;
template <typename E, int kMats, int kI, typename G, typename F>
__device__ inline void few_points(const Product &a, int64_t feature, G ready, F x, typename Ops<E>::Acc (&acc)[kMats][kI])
{
    constexpr int kAtOnce = kI > 1 ? 1 : 4 / kMats; // slices in flight
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();
    const int64_t at = feature + lane % 16, held = at < a.features ? at : a.features - 1;
    const char *row[2] = {a.B + held * a.b_stride, kMats == 2 ? a.B2 + held * a.b2_stride : nullptr};
    Piece q[kAtOnce][kMats][2];
    const auto load = [&](int32_t s0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int32_t s = s0 + u * kFewWaves < a.slices ? s0 + u * kFewWaves : s0; // again, and not used
#pragma unroll
            for (int m = 0; m < kMats; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t k = int64_t(s) * kSlice + h * 64 + lane / 16 * 16;
                    if (int64_t(s + 1) * kSlice <= a.bytes)
                        q[u][m][h] = inner_piece(row[m] + k);
                    else
                        q[u][m][h] = any_piece<E>(row[m], k, a.bytes);
                }
        }
    };
    if (w < a.slices) load(w);
    ready();
    for (int32_t s0 = w; s0 < a.slices;) {
        if constexpr (kI > 1) {
            Piece now[kMats][2], p[2][kI];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kI; ++i) p[h][i] = x(s0, h, i);
#pragma unroll
            for (int m = 0; m < kMats; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) now[m][h] = q[0][m][h];
            s0 += kFewWaves;
            if (s0 < a.slices) load(s0);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < kMats; ++m)
#pragma unroll
                    for (int i = 0; i < kI; ++i) acc[m][i] = Ops<E>::mul(p[h][i], now[m][h], acc[m][i]);
        } else {
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (s0 + u * kFewWaves >= a.slices) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Piece p = x(s0 + u * kFewWaves, h, 0);
#pragma unroll
                    for (int m = 0; m < kMats; ++m) acc[m][0] = Ops<E>::mul(p, q[u][m][h], acc[m][0]);
                }
            }
            s0 += kFewWaves * kAtOnce;
            if (s0 < a.slices) load(s0);
        }
    }
}
// The waves' sums, in order: sum[m] of the block's thread t < 256 for block i of points, of point 16 i + t / 16 and feature t % 16
template <typename V, int kMats, int kI, typename Acc>
__device__ inline void few_put(const Acc (&acc)[kMats][kI], V (*s_sum)[kMats][kI][256])
{
    const int w = int(threadIdx.x) / kWave, lane = lane_id();
#pragma unroll
    for (int m = 0; m < kMats; ++m)
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s_sum[w][m][i][(lane / 16 * 4 + r) * 16 + lane % 16] = acc[m][i][r];
    __syncthreads();
}
template <typename V, int kMats, int kI> __device__ inline V few_sum(const V (*s_sum)[kMats][kI][256], int m, int i, int t)
{
    V sum = V(0);
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) sum += s_sum[k][m][i][t];
    return sum;
}

// ------------------------------------------------------------------ large tiles
// Tiles of 256 x 256 by two groups of four waves, one of each on a SIMD.  A wave's 128 x 64 values are four quarters of
// 64 x 32; a slice takes four steps, one a quarter, and a step has two parts with a barrier behind each: in the first the wave
// reads fragments from LDS and starts its share of the loads, in the second it multiplies (16 blocks of 16 x 16, both halves
// of the slice).  The second group is a part behind the first, so one group's products cover the other's reads.
//
// A slice's four regions (halves of A's and B's rows, 16 KB each) are read in steps 3 (of the slice before), 0, 1 and 2, and
// filled again two steps later, when both groups' reads have been waited for: B0 in step 1, A0 in 2, B1 in 3, A1 in step 0 of the
// next.  So a load has six steps until it is read; a wave waits for its own loads of a region in the first part of the step
// before (loads of five steps, two each, may still be under way), and the barrier behind that is everybody's.
//
// A CU has one such block, which goes on to its next tile: the loads of the last two slices' steps are the next tile's
// first, so they are under way while the outputs are formed and stored.  Rows have two slices at least.
//
// 8192 x 8192 to 8192 at 1.47 PFLOP/s in 16 bits and 2.6 POP/s in 8; matrix cores busy 75 % of the CUs' time at 4096 deep (dx
// of 70000 x 512), 54 % in a product across the rows (8750 points a part).  At 512 to 2048 deep the outputs count, during
// which they rest: 1.0 to 1.3.  (Blocks started apart from each other, by XCD or by CU, so that some would store while others
// multiply: no difference.)
constexpr int kRegion = 128 * kSlice;
constexpr int64_t kLargeStride = int64_t(1) << 23; // bytes
enum class Tail { kWhole, kFirst, kZeros };

//
// Behind the end of K: kWhole, K ends with a slice (kColumns: A has rows of zeros up to there; B's last row is read again and
// cut off in the fragments).  kFirst: A's rows go on with zeros, and B's last piece is read again (integers: zero times any).
// kZeros: both operands' pieces are zeros, by a branch at every load, which costs 10 % (16384 x 8192 to 8192 bf16 3.23 ms a
// pass, without it 2.92).
template <typename E, Form kForm, Tail kTail, typename F> __device__ inline void large_tiles(const Product &a, F finish)
{
    extern __shared__ __align__(16) char s_mem[];
    constexpr bool kDual = kForm == Form::kDual, kColumns = kForm == Form::kColumns;
    constexpr int kEs = int(sizeof(E)), kRowPieces = 128 * kEs / 16; // kColumns: pieces of a region's row
    constexpr int kA0 = 0, kA1 = 1, kB0 = 2, kB1 = 3; // regions
    constexpr int kTogether = kDual ? 2 : 4;
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id(), group = w / 4, column = w % 4;
    const int32_t first = int32_t(blockIdx.y) * a.per_split;
    const int32_t slices = (first + a.per_split < a.slices ? first + a.per_split : a.slices) - first;
    const uint32_t tiles = uint32_t(a.down) * uint32_t(a.across);
    const int own = ((lane % 8) ^ (lane / 8)) * 16;
    const int row0 = (w * kWave + lane) / kRowPieces, piece0 = (w * kWave + lane) % kRowPieces; // kColumns: of the first of two
    // of the row (of the column), from this lane's first piece on
    const int64_t left = a.bytes - int64_t(first) * kSlice - (kColumns ? row0 * kEs : own);
    const int64_t a_step = kColumns ? kSlice / kEs * a.a_stride : kSlice, b_step = kColumns ? kSlice / kEs * a.b_stride : kSlice;

    // Regions' rows: A's half h has the h-th 64 of each group's 128 points, B's the blocks 2 h and 2 h + 1 of each column of
    // waves.  This lane's pieces of the two kilobytes that the wave loads of each region: where they lie behind the tile's
    // first value, in 32 bits (strides are kLargeStride at most), so that the addresses' high parts stay in scalar registers.
    const char *base[4];
    uint32_t off[4][2];
    const auto point = [&](int r, int32_t bi, int32_t bj) {
        const int h = r & 1;
        const bool of_a = r < kB0, second = kDual && !of_a && h == 1;
        const int64_t stride = of_a ? a.a_stride : second ? a.b2_stride : a.b_stride;
        const int64_t tile = int64_t(of_a ? bi : bj) * (kDual && !of_a ? 128 : 256), most = (of_a ? a.rows : a.features) - tile; // values left
        base[r] = (of_a ? a.A : second ? a.B2 : a.B) + (kColumns ? tile * kEs + int64_t(first) * (kSlice / kEs) * stride : tile * stride + int64_t(first) * kSlice);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if constexpr (kColumns) {
                const int row = row0 + e * (8 * kWave / kRowPieces), value = column_piece<E, 128 * kEs>(piece0, row) * (16 / kEs);
                const int at = of_a ? value / 64 * 128 + h * 64 + value % 64 : value / 32 * 64 + h * 32 + value % 32, last = 16 / kEs;
                off[r][e] = uint32_t(row) * uint32_t(stride) + uint32_t(at + last <= most ? at : int(most) - last) * kEs;
            } else {
                const int row = (e * 8 + w) * 8 + lane / 8, i = row % 16, block = row % 32 / 16; // of the region
                const int at = of_a ? row / 64 * 128 + h * 64 + row % 64
                                    : row / 32 * (16 * kTogether) + i * kTogether + (second ? block : 2 * h + block);
                off[r][e] = uint32_t(at < most ? at : int(most) - 1) * uint32_t(stride) + uint32_t(own);
            }
        }
    };
    // region r of a slice into the buffers of its parity
    const int32_t rest = int32_t(a.bytes - int64_t(first) * kSlice < (int64_t(1) << 30) ? a.bytes - int64_t(first) * kSlice : int64_t(1) << 30);
    const auto fetch = [&](int r, int32_t slice, int parity) {
        char *to = s_mem + parity * (4 * kRegion) + r * kRegion;
        const char *from = base[r] + slice * (r < kB0 ? a_step : b_step);
        const auto load = [&](const char *p, int e) {
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p,
                                             (__attribute__((address_space(3))) void *)(to + (e * 8 + w) * 8 * kSlice), 16, 0, 0);
        };
        if (kTail == Tail::kZeros && int64_t(slice + 1) * kSlice > int64_t(rest)) {
#pragma unroll
            for (int e = 0; e < 2; ++e) load(left - int64_t(slice) * kSlice <= 0 ? kZeros : from + off[r][e], e);
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint32_t o = off[r][e];
                if constexpr (kTail == Tail::kFirst) {
                    const int over = slice * kSlice + own - (rest - 16); // bytes behind the last piece
                    if (r >= kB0) o -= uint32_t(over > 0 ? over : 0);
                }
                if constexpr (kColumns) {
                    const int over = (slice * kSlice - rest) / kEs + 1 + row0 + e * (8 * kWave / kRowPieces); // rows behind the last one
                    if (r >= kB0) o -= uint32_t(over > 0 ? over : 0) * uint32_t(a.b_stride);
                }
                load(from + o, e);
            }
        }
    };
    const int at0 = lane % 16 * kSlice + ((lane / 16) ^ (lane & 7)) * 16, at1 = at0 ^ 64; // the two halves of a slice
    Piece p[2][4], q[2][2][2]; // A's half that is under way; both of B's
    // kColumns: the lane's places in this slice's buffers
    const char *in_a[4], *in_b[2];
    if constexpr (kColumns) {
#pragma unroll
        for (int i = 0; i < 4; ++i) in_a[i] = s_mem + column_place<E, 128 * kEs>(group * 4 + i);
#pragma unroll
        for (int j = 0; j < 2; ++j) in_b[j] = s_mem + column_place<E, 128 * kEs>(column * 2 + j);
    }
    const auto read_a = [&](int h, int parity) {
        if constexpr (kColumns) {
            if (h)
                column_slices<E, 128 * kEs, kRegion>(in_a, p);
            else
                column_slices<E, 128 * kEs, 0>(in_a, p);
            return;
        }
        const char *in = s_mem + parity * (4 * kRegion) + h * kRegion + group * 64 * kSlice;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[0][i] = *reinterpret_cast<const Piece *>(in + i * 16 * kSlice + at0);
            p[1][i] = *reinterpret_cast<const Piece *>(in + i * 16 * kSlice + at1);
        }
    };
    const auto read_b = [&](int h, int parity, bool ahead = false) {
        if constexpr (kColumns) {
            const int by = ahead ? (parity ? 4 : -4) * kRegion : 0;
            const char *const at[2] = {in_b[0] + by, in_b[1] + by};
            if (h)
                column_slices<E, 128 * kEs, kB1 * kRegion>(at, q[1]);
            else
                column_slices<E, 128 * kEs, kB0 * kRegion>(at, q[0]);
            return;
        }
        const char *in = s_mem + parity * (4 * kRegion) + (kB0 + h) * kRegion + column * 32 * kSlice;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            q[h][0][j] = *reinterpret_cast<const Piece *>(in + j * 16 * kSlice + at0);
            q[h][1][j] = *reinterpret_cast<const Piece *>(in + j * 16 * kSlice + at1);
        }
    };
    typename Ops<E>::Acc acc[8][4];
    // the barrier between a step's parts, with the wait for the loads that the next step reads; and the part that multiplies
    const auto multiply = [&](int ha, int hb, int32_t slice) {
        asm volatile("s_waitcnt vmcnt(10)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (kColumns) {
            const int rows = (rest - slice * kSlice) / kEs; // of this slice
            if (rows < kSlice / kEs) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (kEs == 2) {
                                const int more = rows - 32 * half - lane / 16 * 8 - 2 * e; // of two
                                q[hb][half][j][e] = more >= 2 ? q[hb][half][j][e] : more == 1 ? q[hb][half][j][e] & 0xffff : 0;
                            } else {
                                q[hb][half][j][e] = 16 * half + 4 * e + lane / 16 < rows ? q[hb][half][j][e] : 0;
                            }
                        }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[4 * ha + i][2 * hb + j] = Ops<E>::mul(p[half][i], q[hb][half][j], acc[4 * ha + i][2 * hb + j]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    uint32_t t = blockIdx.x;
    int32_t bi, bj;
    place(a, t, bi, bj);
#pragma unroll
    for (int r = 0; r < 4; ++r) point(r, bi, bj);
    fetch(kB0, 0, 0);
    fetch(kA0, 0, 0);
    fetch(kB1, 0, 0);
    fetch(kA1, 0, 0);
    fetch(kB0, 1, 1);
    fetch(kA0, 1, 1);
    fetch(kB1, 1, 1);
    asm volatile("s_waitcnt vmcnt(10)\n\ts_barrier" ::: "memory");
    int parity = 0;
    for (;;) {
        const uint32_t next = t + gridDim.x;
        const bool more = next < tiles; // without, the last loads are this tile's first again, which nobody reads
        int32_t ni = bi, nj = bj;
        if (more) place(a, next, ni, nj);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = {};
        read_b(0, parity);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // the first group fills this region again in its step 1
        if (group == 1) asm volatile("s_barrier" ::: "memory"); // a part behind
        __builtin_amdgcn_sched_barrier(0);
        for (int32_t slice = 0; slice < slices; ++slice, parity ^= 1) {
            const int32_t one = slice + 1 < slices ? slice + 1 : 0, two = slice + 2 < slices ? slice + 2 : slice + 2 - slices;
            if (slice == slices - 1) point(kA1, ni, nj);
            read_a(0, parity);
            fetch(kA1, one, parity ^ 1);
            multiply(0, 0, slice);
            if (slice == slices - 2) {
                point(kB0, ni, nj);
                point(kA0, ni, nj);
                point(kB1, ni, nj);
            }
            read_b(1, parity);
            fetch(kB0, two, parity);
            multiply(0, 1, slice);
            read_a(1, parity);
            fetch(kA0, two, parity);
            multiply(1, 0, slice);
            read_b(0, parity ^ 1, true); // behind the tile's last slice: the next one's, read again
            fetch(kB1, two, parity);
            multiply(1, 1, slice);
            if constexpr (kColumns) {
                const int flip = parity ? -4 * kRegion : 4 * kRegion;
#pragma unroll
                for (int i = 0; i < 4; ++i) in_a[i] += flip;
#pragma unroll
                for (int j = 0; j < 2; ++j) in_b[j] += flip;
            }
        }
        if (group == 0) asm volatile("s_barrier" ::: "memory"); // the groups meet, so that both form their outputs at once
        __builtin_amdgcn_sched_barrier(0);
        finish(bi, bj, acc);
        if (!more) break;
        t = next;
        bi = ni;
        bj = nj;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); // no load is under way when the block's LDS is given on
}

// The tiles of a launch: finish(bi, bj, acc) takes each one's sums
template <typename E, typename T, Form kForm, bool kAny, Tail kTail, typename F> __device__ inline void each_tile(const Product &a, F finish)
{
    if constexpr (std::is_same<T, TileLarge>::value) {
        large_tiles<E, kForm, kTail>(a, finish);
    } else {
        int32_t bi, bj;
        place(a, blockIdx.x, bi, bj);
        typename Ops<E>::Acc acc[T::kI][T::kJ] = {};
        multiply_tile<E, T, kForm, kAny>(a, bi, bj, acc);
        finish(bi, bj, acc);
    }
}
template <typename T> inline uint32_t blocks_of(uint32_t tiles)
{
    return std::is_same<T, TileLarge>::value && tiles > uint32_t(kCus) ? uint32_t(kCus) : tiles;
}

// Points and features of a lane: f(point, feature, i, r) for row r of each block i of points, with the lane's first
// feature, of kTogether consecutive ones: acc[i][..][r].  kColumns: features 16 apart.
template <typename T, Form kForm, typename F> __device__ inline void each_run(int32_t bi, int32_t bj, F f)
{
    constexpr int kTogether = kForm == Form::kDual ? T::kJ / 2 : T::kJ;
    const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();
    const int64_t feature = int64_t(bj) * (kForm == Form::kDual ? T::kN / 2 : T::kN) + w % T::kWn * (16 * kTogether)
                            + lane % 16 * (kForm == Form::kColumns ? 1 : kTogether);
    const int64_t point = int64_t(bi) * T::kM + w / T::kWn * (T::kI * 16) + lane / 16 * 4;
#pragma unroll
    for (int i = 0; i < T::kI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) f(point + 16 * i + r, feature, i, r);
}

// An output of the value: rounded from 32 bits.  In fp16 the compiler rounds some products once, from all of their bits, and
// others not; what is stored is not to depend on which.
template <typename E> __device__ inline E rounded(float v)
{
    if constexpr (std::is_same<E, f16>::value) asm("" : "+v"(v));
    return E(v);
}

// N consecutive values to p, of which `count` exist; vec: aligned to 16 bytes, or to N values where those are less
template <typename E, int N> __device__ inline void store_run(E *p, const float (&v)[N], int64_t count, bool vec)
{
    constexpr int kV = 16 / int(sizeof(E)) < N ? 16 / int(sizeof(E)) : N;
    struct alignas(sizeof(E) * kV) Pack {
        E v[kV];
    };
    if (vec && count >= N) {
#pragma unroll
        for (int h = 0; h < N / kV; ++h) {
            Pack x;
#pragma unroll
            for (int e = 0; e < kV; ++e) x.v[e] = rounded<E>(v[h * kV + e]);
            reinterpret_cast<Pack *>(p)[h] = x;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < count) p[e] = rounded<E>(v[e]);
}

// Tiles inside the output whose runs are vectors: a run's place is the wave's, the same for all lanes, and one 32-bit offset of
// the lane's for all rows (strides are kLargeStride at most).  With each run's own 64-bit place, count and branches a tile of
// 256 x 256 took 5 us more (16384 x 2048 to 8192 bf16, with three outputs, 914 us for 836; 70001 x 2000 to 2000 in 8 bits 445
// for 400).
template <typename T, Form kForm> __device__ inline bool tile_inside(const Product &a, int32_t bi, int32_t bj)
{
    constexpr int kN = kForm == Form::kDual ? T::kN / 2 : T::kN;
    return int64_t(bi) * T::kM + T::kM <= a.rows && int64_t(bj) * kN + kN <= a.features;
}
template <typename T, Form kForm> struct InnerRuns {
    static constexpr int kTogether = kForm == Form::kDual ? T::kJ / 2 : T::kJ;
    int64_t row, feature; // the wave's first
    uint32_t lane_row, lane_feature;
    __device__ inline InnerRuns(int32_t bi, int32_t bj)
    {
        const int w = int(uniform(threadIdx.x / kWave)), lane = lane_id();
        row = int64_t(bi) * T::kM + w / T::kWn * (T::kI * 16);
        feature = int64_t(bj) * (kForm == Form::kDual ? T::kN / 2 : T::kN) + w % T::kWn * (16 * kTogether);
        lane_row = uint32_t(lane / 16 * 4);
        lane_feature = uint32_t(lane % 16 * kTogether);
    }
    // kTogether values of the lane's point 16 i + r
    template <typename E> struct To {
        char *first;
        int64_t stride; // bytes
        uint32_t lane;
        __device__ inline void put(int i, int r, const float (&v)[kTogether]) const
        {
            constexpr int kV = 16 / int(sizeof(E)) < kTogether ? 16 / int(sizeof(E)) : kTogether;
            struct alignas(sizeof(E) * kV) Pack {
                E v[kV];
            };
#pragma unroll
            for (int h = 0; h < kTogether / kV; ++h) {
                Pack x;
#pragma unroll
                for (int e = 0; e < kV; ++e) x.v[e] = rounded<E>(v[h * kV + e]);
                *reinterpret_cast<Pack *>(first + (16 * i + r) * stride + lane + h * sizeof(Pack)) = x;
            }
        }
    };
    template <typename E> __device__ inline To<E> to(void *out, int64_t stride) const
    {
        const int64_t s = stride * int64_t(sizeof(E));
        return {static_cast<char *>(out) + row * s + feature * int64_t(sizeof(E)), s, lane_row * uint32_t(s) + lane_feature * uint32_t(sizeof(E))};
    }
};

inline bool aligned_to(int bytes, const void *p, int64_t stride_bytes)
{
    return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0 && stride_bytes % bytes == 0;
}
inline bool aligned16(const void *p, int64_t stride_bytes) { return aligned_to(16, p, stride_bytes); }
// whether store_run's vectors of N values can be used
template <typename E, int N> inline bool runs_aligned(const void *p, int64_t stride)
{
    constexpr int kBytes = int(sizeof(E)) * N;
    return aligned_to(kBytes < 16 ? kBytes : 16, p, stride * int64_t(sizeof(E)));
}

// ... and InnerRuns: no output is such, too
template <typename E, int N> inline bool runs_inner(const void *p, int64_t stride)
{
    return !p || (runs_aligned<E, N>(p, stride) && stride * int64_t(sizeof(E)) <= kLargeStride);
}

inline int64_t slices_of(int64_t bytes) { return (bytes + kSlice - 1) / kSlice; }

// A launch takes at most kMostTiles tiles: rows are cut into several launches beyond
constexpr int64_t kMostTiles = int64_t(1) << 22;

} // namespace prod
} // namespace bht
