// Matrix products on tiles of 32 x 32 with the contraction in steps of 16, for fp16, bf16 and fp32 operands and
// fp32 sums.
//
// Every operator here has one side that stays in registers (32 columns, one a lane of each half wave) and streams
// the other through LDS, twice over: once by rows (a product over the row's elements gives scores, 32 streamed rows
// by 32 columns) and once by columns (a product over the streamed rows, with what became of the scores).
//   A (streamed): lane l holds row l & 31, elements k = (l >> 5) * 8 .. + 8 of the step
//   B (kept):     lane l holds column l & 31, the same elements k
//   sums:         lane l holds column l & 31, register r holds row 8 * (r >> 2) + 4 * (l >> 5) + (r & 3)
// The second product contracts over the streamed rows in the order in which the sums' registers hold them, so the
// scores go from sums to B without leaving their lane: step m takes registers 8m .. 8m + 7.  16-bit columns are read
// by the LDS's transposing loads, which hand a lane four rows of its column.
// Which streamed row stands in which row of the product is free.  Rows lie an odd multiple of 4 banks (of 64, 4 bytes
// each) apart by 16 bytes of padding, which suits the reads by rows, 16 bytes from each of 16 rows at a time; the
// transposing reads take 64 bytes from each of 4 rows at a time, which must lie 4 rows apart not to meet.  So rows
// 0 .. 3 of the product are rows 0, 4, 8, 12 of the tile, and so on (recd_tile_row).  With rows in order 56 % of the LDS's
// busy cycles were conflicts, with rows two apart 30 %, so none.
#pragma once

#include "recd_vec.h"

typedef float recd_f32x16 __attribute__((ext_vector_type(16)));
typedef float recd_f32x8 __attribute__((ext_vector_type(8)));
typedef short recd_s16x4 __attribute__((ext_vector_type(4)));

template <typename T> struct RecdMma;

template <> struct RecdMma<_Float16> {
    using Frag = recd_f16x8;
    static __device__ inline recd_f32x16 mul(Frag a, Frag b, recd_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct RecdMma<__bf16> {
    using Frag = recd_bf16x8;
    static __device__ inline recd_f32x16 mul(Frag a, Frag b, recd_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct RecdMma<float> {
    using Frag = recd_f32x8;
    // step e contracts element e of the lower half wave's eight and of the upper's
    static __device__ inline recd_f32x16 mul(Frag a, Frag b, recd_f32x16 c)
    {
#pragma unroll
        for (int e = 0; e < 8; e++)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// The tile's row (of 32) in row i of the product.
__device__ inline int recd_tile_row(int i) { return (i & 16) | (i & 3) << 2 | (i >> 3 & 1) << 1 | (i >> 2 & 1); }
// The row of the product that tile row i stands in.
__device__ inline int recd_product_row(int i) { return (i & ~15) | (i >> 1 & 1) << 3 | (i & 1) << 2 | (i >> 2 & 3); }
// Row of the product in a sums' register, and the tile's row in a score's.
__device__ inline int recd_sums_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }
__device__ inline int recd_score_row(int r, int lane) { return 16 * (r >> 3) + 4 * (r & 3) + 2 * (r >> 2 & 1) + (lane >> 5); }

// 0 * x is a NaN where x is an infinity or a NaN: an operation a word, of one or two values, and `sum` stays 0 without them.
typedef _Float16 recd_f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 recd_bf16x2 __attribute__((ext_vector_type(2)));
template <typename T> __device__ inline float recd_zeros(typename RecdPiece<T>::type v, float sum)
{
    const recd_u32x4 b = __builtin_bit_cast(recd_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (sizeof(T) == 4)
            sum = __builtin_fmaf(v[i], 0.0f, sum);
        else if constexpr (std::is_same<T, _Float16>::value)
            sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(recd_f16x2, (uint32_t)b[i]), recd_f16x2{}, sum, false);
        else
            sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(recd_bf16x2, (uint32_t)b[i]), recd_bf16x2{}, sum, false);
    }
    return sum;
}
// Infinities and NaN are the values whose exponent is all ones: one more carries into the sign's place.
template <typename T> struct RecdExponent {
    static constexpr bool HALF = std::is_same<T, _Float16>::value;
    static constexpr uint32_t ALL = sizeof(T) == 4 ? 0x7f800000u : HALF ? 0x7c007c00u : 0x7f807f80u;
    static constexpr uint32_t ONE = sizeof(T) == 4 ? 0x00800000u : HALF ? 0x04000400u : 0x00800080u;
    static constexpr uint32_t SIGN = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    static constexpr int TOP = sizeof(T) == 4 ? 31 : 15;
};
// The piece with zeros in their place.
template <typename T> __device__ inline typename RecdPiece<T>::type recd_finite(typename RecdPiece<T>::type v)
{
    using X = RecdExponent<T>;
    recd_u32x4 b = __builtin_bit_cast(recd_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t hit = ((b[i] & X::ALL) + X::ONE) & X::SIGN;
        b[i] &= ~((hit - (hit >> X::TOP)) | hit);
    }
    return __builtin_bit_cast(typename RecdPiece<T>::type, b);
}

// A tile of ROWS rows of DP elements in LDS.
template <typename T, int ROWS, int DP> struct RecdTile {
    static constexpr int E = 16 / sizeof(T), LD = DP + E, PIECES = ROWS * (DP / E);
    using Frag = typename RecdMma<T>::Frag;
    using Piece = typename RecdPiece<T>::type;
    alignas(16) T at[ROWS * LD];

    // elements k0 .. k0 + 16 of the 32 rows from row0 on
    __device__ inline Frag rows(int row0, int k0, int lane) const
    {
        return *reinterpret_cast<const Frag *>(at + (row0 + recd_tile_row(lane & 31)) * LD + k0 + (lane >> 5) * 8);
    }
    // columns d0 .. d0 + 32 of the 16 rows from row0 on, in the order of the sums' registers
    __device__ inline Frag columns(int row0, int d0, int lane) const
    {
        if constexpr (sizeof(T) == 4) {
            Frag f;
            const T *p = at + (row0 + (lane >> 5)) * LD + d0 + (lane & 31);
#pragma unroll
            for (int e = 0; e < 8; e++)
                f[e] = p[(2 * (e >> 2) + 4 * (e & 3)) * LD];
            return f;
        } else {
            // 16 lanes name four rows of 16 columns, 8 bytes each; each of them receives one column
            using Half = __attribute__((address_space(3))) recd_s16x4;
            const int i = lane & 15;
            const T *p = at + (row0 + (lane >> 5) + 4 * (i >> 2)) * LD + d0 + 16 * ((lane >> 4) & 1) + 4 * (i & 3);
            union {
                recd_s16x4 half[2];
                Frag f;
            } u;
            u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half *)(p));
            u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Half *)(p + 2 * LD));
            return u.f;
        }
    }
    __device__ inline void put_at(int row, int column, Piece v) { *reinterpret_cast<Piece *>(at + row * LD + column) = v; }
    __device__ inline void put(int piece, Piece v)
    {
        constexpr int PR = DP / E;
        put_at(piece / PR, piece % PR * E, v);
    }
    // zeros in the place of all that is not finite, by `threads` threads of which this is `tid`, each in the pieces that it puts
    __device__ inline void make_finite(int tid, int threads)
    {
        constexpr int PR = DP / E;
        asm volatile("" : "+v"(tid));  // nothing of this is held in registers before it is needed
#pragma unroll 1
        for (int piece = tid; piece < PIECES; piece += threads)
            put(piece, recd_finite<T>(*reinterpret_cast<const Piece *>(at + (piece / PR) * LD + (piece % PR) * E)));
    }
};

// Rows of a tile from memory into registers and on into LDS, by THREADS threads of which this is `tid`.  A thread's
// addresses are 32-bit offsets from the tile's first row, which is the same for all: bytes(r) is that of row r < 128.  Rows
// behind the last one and elements behind a row's last one are read from the last one's place instead.  The scores of such
// rows are masked; such elements go to the padding behind a tile's rows, and zeros stand in their place (clear_behind), as in the
// kept operand: an infinity against that one's zeros would turn the sum of the others into a NaN.
template <typename T, int ROWS, int DP, int THREADS> struct RecdStream {
    using Tile = RecdTile<T, ROWS, DP>;
    using Piece = typename Tile::Piece;
    static constexpr int PT = (Tile::PIECES + THREADS - 1) / THREADS;
    Piece held[PT];

    template <typename Bytes> __device__ inline void load(int tid, const T *first, int rows, int d, Bytes bytes)
    {
        constexpr int PR = DP / Tile::E;
#pragma unroll
        for (int i = 0; i < PT; i++) {
            const int piece = tid + i * THREADS, at = piece % PR * Tile::E, r = piece / PR;
            if (piece < Tile::PIECES) {
                const uint32_t off = bytes(r < rows ? r : rows - 1) + (uint32_t)((at < d ? at : d - Tile::E) * (int)sizeof(T));
                held[i] = *reinterpret_cast<const Piece *>(reinterpret_cast<const char *>(first) + off);
            }
        }
    }
    // rows that lie `stride` bytes (less than 2^24) apart
    __device__ inline void load_rows(int tid, const T *first, int rows, int d, uint32_t stride)
    {
        load(tid, first, rows, d, [=](int r) { return (uint32_t)__umul24(r, stride); });
    }
    // whether the thread's pieces hold anything that is not finite
    __device__ inline bool not_finite(int tid) const
    {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PT; i++)
            if (tid + i * THREADS < Tile::PIECES)
                sum = recd_zeros<T>(held[i], sum);
        return !(sum == 0.0f);
    }
    // the tile's row of a thread's piece i
    static __device__ inline int row(int tid, int i) { return (tid + i * THREADS) / (DP / Tile::E); }
    __device__ inline void store(int tid, Tile &t, int d)
    {
#pragma unroll
        for (int i = 0; i < PT; i++)
            if (tid + i * THREADS < Tile::PIECES)
                t.put_at((tid + i * THREADS) / (DP / Tile::E), column(tid, i) < d ? column(tid, i) : DP, held[i]);
    }
    // zeros behind the rows' d elements, which stay there, in the places where the thread would put pieces
    static __device__ inline void clear_behind(int tid, Tile &t, int d)
    {
#pragma unroll
        for (int i = 0; i < PT; i++)
            if (tid + i * THREADS < Tile::PIECES && column(tid, i) >= d)
                t.put(tid + i * THREADS, Piece{});
    }
    // the first element of a thread's piece i
    static __device__ inline int column(int tid, int i)
    {
        constexpr int PR = DP / Tile::E;
        return (THREADS % PR == 0 ? tid : tid + i * THREADS) % PR * Tile::E;
    }
};

// What the wave's lanes wrote to LDS is there for its other lanes; what they read has been read.
__device__ inline void recd_wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The step's 16 elements from k0 on of a row in global memory (8 a half wave), zero from element D on.
template <typename T> __device__ inline typename RecdMma<T>::Frag recd_row_frag(const T *row, int k0, int D, bool there, int lane)
{
    constexpr int E = 16 / sizeof(T);
    union {
        typename RecdPiece<T>::type piece[8 / E];
        typename RecdMma<T>::Frag f;
    } u;
#pragma unroll
    for (int i = 0; i < 8 / E; i++) {
        const int k = k0 + (lane >> 5) * 8 + i * E;
        u.piece[i] = typename RecdPiece<T>::type{};
        if (there && k < D)
            u.piece[i] = *reinterpret_cast<const typename RecdPiece<T>::type *>(row + k);
    }
    return u.f;
}

template <typename Frag> __device__ inline Frag recd_negated(Frag f)
{
#pragma unroll
    for (int e = 0; e < 8; e++)
        f[e] = -f[e];
    return f;
}

// Sums' registers 8m .. 8m + 7 as the B operand of a product over streamed rows.
template <typename T> __device__ inline typename RecdMma<T>::Frag recd_sums_frag(const recd_f32x16 &s, int m)
{
    typename RecdMma<T>::Frag f;
#pragma unroll
    for (int e = 0; e < 8; e++)
        f[e] = (T)s[8 * m + e];
    return f;
}

constexpr float kRecdLog2e = 1.4426950408889634f, kRecdLn2 = 0.6931471805599453f;
__device__ inline float recd_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The tiles' width for rows of D elements.
template <typename F> void recd_with_width(int D, F f)
{
    if (D <= 32)
        f(std::integral_constant<int, 32>{});
    else if (D <= 64)
        f(std::integral_constant<int, 64>{});
    else if (D <= 96)
        f(std::integral_constant<int, 96>{});
    else if (D <= 128)
        f(std::integral_constant<int, 128>{});
    else if (D <= 192)
        f(std::integral_constant<int, 192>{});
    else
        f(std::integral_constant<int, 256>{});
}
