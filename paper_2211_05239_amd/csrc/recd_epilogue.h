// What becomes of a row's elements on their way out of a product's sums: bias, activation, dropout, residual, and the
// gradients of these.  Eight neighbouring columns of a row at a time, in 32 bits.
#pragma once

#include "recd_internal.h"
#include "recd_vec.h"

// ---- dropout -----------------------------------------------------------------------------------------------------
// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011) of the key `seed`
// and the counter (column / 8 | row's upper bits, row, call): 16 of its 128 bits for each of eight neighbours, and an
// element stays where they are not below `cut` = p * 2^16.  The mask of a place is the same in every kernel and both
// directions, and is never stored.  With 32 bits an element the generator would take twice the products (20 of 32 x 32
// bits for eight elements now, a quarter of the vector units' rate each); a p between the steps of 2^-16 is rounded to one
// and the kept elements are scaled for the rounded one, so the expected value is exact.
struct RecdMask {
    uint32_t k0, k1, cut;
    float by;
    uint64_t call;
    const int64_t *step;
};

constexpr int RECD_MAX_WIDTH = 65536;  // of a row that has a mask or goes through a layer

// Checks the mask a caller describes and brings it into the kernels' form; no mask: cut = 0.
recd_status recd_make_mask(recd_ctx *ctx, const recd_dropout_mask *m, RecdMask *out);

struct RecdBits {
    uint32_t w[4];
    __device__ inline bool keep(int e, uint32_t cut) const { return ((e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) >= cut; }
};

// The call's number, with what the device adds to it.
__device__ inline uint64_t recd_mask_call(const RecdMask &m) { return m.step ? m.call + (uint64_t)*m.step : m.call; }

__device__ inline void recd_philox(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d, uint32_t k0, uint32_t k1)
{
    const uint64_t u = (uint64_t)a * 0xD2511F53u, v = (uint64_t)c * 0xCD9E8D57u;
    a = __builtin_amdgcn_bitop3_b32((uint32_t)(v >> 32), b, k0, 0x96);  // xor of the three
    b = (uint32_t)v;
    c = __builtin_amdgcn_bitop3_b32((uint32_t)(u >> 32), d, k1, 0x96);
    d = (uint32_t)u;
}

// What a column's piece has of the first three rounds in all rows below 2^32: of their six products the rows need two.  The state (a, b, c, d)
// begins as (piece, row, call); a of the second round and c of the third follow from the row alone or from both, the others from the piece.
// (Both directions of a layer 128 -> 512 with GELU and dropout on 300 007 rows: 600 us without it, 594 with it, and 584 where the
// rows of a lane are made beside each other besides.)
struct RecdMaskPiece {
    uint32_t a1, d1, b2, c3, d3;  // a1 without the row, c3 without d2
};

__device__ inline RecdMaskPiece recd_mask_piece(const RecdMask &m, uint64_t call, int piece)
{
    const uint64_t u1 = (uint64_t)(uint32_t)piece * 0xD2511F53u, v1 = (uint64_t)(uint32_t)call * 0xCD9E8D57u;
    const uint32_t c1 = (uint32_t)(u1 >> 32) ^ (uint32_t)(call >> 32) ^ m.k1;
    const uint64_t v2 = (uint64_t)c1 * 0xCD9E8D57u;
    const uint32_t a2 = (uint32_t)(v2 >> 32) ^ (uint32_t)v1 ^ (m.k0 + 0x9E3779B9u);
    const uint64_t u3 = (uint64_t)a2 * 0xD2511F53u;
    return RecdMaskPiece{(uint32_t)(v1 >> 32) ^ m.k0, (uint32_t)u1, (uint32_t)v2, (uint32_t)(u3 >> 32) ^ (m.k1 + 2 * 0xBB67AE85u), (uint32_t)u3};
}

__device__ inline RecdBits recd_mask_bits(const RecdMask &m, const RecdMaskPiece &p, uint32_t row)
{
    const uint64_t u2 = (uint64_t)(p.a1 ^ row) * 0xD2511F53u;
    const uint32_t c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(u2 >> 32), p.d1, m.k1 + 0xBB67AE85u, 0x96);
    const uint64_t v3 = (uint64_t)c2 * 0xCD9E8D57u;
    uint32_t a = __builtin_amdgcn_bitop3_b32((uint32_t)(v3 >> 32), p.b2, m.k0 + 2 * 0x9E3779B9u, 0x96);
    uint32_t b = (uint32_t)v3, c = p.c3 ^ (uint32_t)u2, d = p.d3;
#pragma unroll
    for (uint32_t i = 3; i < 10; i++)
        recd_philox(a, b, c, d, m.k0 + i * 0x9E3779B9u, m.k1 + i * 0xBB67AE85u);
    return RecdBits{{a, b, c, d}};
}

__device__ inline RecdBits recd_mask_bits(const RecdMask &m, uint64_t call, int64_t row, int piece)
{
    uint32_t a = (uint32_t)piece + ((uint32_t)(row >> 32) << 16), b = (uint32_t)row, c = (uint32_t)call, d = (uint32_t)(call >> 32);
#pragma unroll
    for (uint32_t i = 0; i < 10; i++)
        recd_philox(a, b, c, d, m.k0 + i * 0x9E3779B9u, m.k1 + i * 0xBB67AE85u);
    return RecdBits{{a, b, c, d}};
}

// 0 (also for an infinity or a NaN) where an element does not stay.
__device__ inline void recd_mask_drop(const RecdMask &m, const RecdBits &bits, float *v)
{
#pragma unroll
    for (int e = 0; e < 8; e++)
        v[e] = bits.keep(e, m.cut) ? v[e] : 0.0f;
}

// v times 1 / (1 - p) where it stays, 0 where it does not.
__device__ inline void recd_mask_apply(const RecdMask &m, const RecdBits &bits, float *v)
{
#pragma unroll
    for (int e = 0; e < 8; e++)
        v[e] *= m.by;
    recd_mask_drop(m, bits, v);
}

// ---- activations -------------------------------------------------------------------------------------------------
// GELU is z * P(z) with the normal distribution's P.  For a >= 0, P(-a) = exp(-a^2 / 2) * t * poly(t), t = 1 / (1 + 0.3 a): a
// polynomial of degree 7, fitted to erfcx(a / sqrt(2)) / 2 / t over a in [0, 14.5], where it is off by 1.7e-7 of the value.  In 32 bits
// P(-a) is off by 9e-7 of itself up to a = 4, beyond by what a^2's rounding leaves of the exponential.  No cancellation on
// either side, and the slope P(z) + z exp(-z^2 / 2) / sqrt(2 pi) shares the exponential.
struct RecdNormal {
    float P, e;  // P(z), exp(-z^2 / 2)
};

__device__ inline RecdNormal recd_normal(float z)
{
    const float a = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.0f));
    float p = 0.03542371094226837f;
    p = __builtin_fmaf(p, t, -0.15615835785865784f);
    p = __builtin_fmaf(p, t, 0.2045566290616989f);
    p = __builtin_fmaf(p, t, -0.05203389376401901f);
    p = __builtin_fmaf(p, t, 0.12769171595573425f);
    p = __builtin_fmaf(p, t, 0.10017596185207367f);
    p = __builtin_fmaf(p, t, 0.12071213126182556f);
    p = __builtin_fmaf(p, t, 0.11963200569152832f);
    const float e = __builtin_amdgcn_exp2f(z * z * -0.7213475204444817f);
    p = p * t * e;
    return {z < 0.0f ? p : 1.0f - p, e};
}

__device__ inline float recd_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }

// v[e] = act(v[e]); `act` is the same for all lanes.
__device__ inline void recd_activate(int act, float *v)
{
    if (act == RECD_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            v[e] = v[e] <= 0.0f ? 0.0f : v[e];  // (a NaN stays)
    } else if (act == RECD_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            v[e] *= recd_normal(v[e]).P;
    } else if (act == RECD_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            v[e] *= recd_sigmoid(v[e]);
    }
}

// g[e] *= act'(z[e]).  ReLU's slope at 0 is 0.
__device__ inline void recd_activate_back(int act, const float *z, float *g)
{
    if (act == RECD_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            g[e] = z[e] <= 0.0f ? 0.0f : g[e];
    } else if (act == RECD_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const RecdNormal n = recd_normal(z[e]);
            g[e] *= __builtin_fmaf(z[e] * 0.3989422804014327f, n.e, n.P);
        }
    } else if (act == RECD_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float s = recd_sigmoid(z[e]);
            g[e] *= s * (1.0f + z[e] * (1.0f - s));
        }
    }
}

// ---- rows' elements, eight at a time -------------------------------------------------------------------------------
// The first `count` (8, or 4 at the end of a row of 4-byte elements) of the eight elements at p, aligned to 16 bytes.
template <typename T> __device__ inline void recd_load8(const T *p, int count, float *v)
{
    recd_load16(p, v);
    if constexpr (sizeof(T) == 4) {
        if (count == 8)
            recd_load16(p + 4, v + 4);
        else
#pragma unroll
            for (int e = 4; e < 8; e++)
                v[e] = 0.0f;
    }
}

template <typename T> __device__ inline void recd_store8(T *p, int count, const float *v)
{
    recd_store16(p, v);
    if constexpr (sizeof(T) == 4)
        if (count == 8)
            recd_store16(p + 4, v + 4);
}

// The same past the caches' retention for 16-bit elements: what a kernel writes once and reads no more.  A die's L2 hands it on at the
// kernel's end at the latest, so that a later reader loses nothing, and what the kernel reads keeps its place (300 007 x 128 -> 512 bf16
// 140 -> 118 us, 512 -> 128's gradient by x 108 -> 90, dropout and its gradient of 300 007 x 128 84 -> 76).  A lane's eight 32-bit elements
// are two stores 32 bytes from lane to lane, half lines that have to wait for each other in the L2 (dropout of 50 021 x 516 97 -> 127).
template <typename T> __device__ inline void recd_store8_past(T *p, int count, const float *v)
{
    if constexpr (sizeof(T) == 4)
        recd_store8(p, count, v);
    else {
        typename RecdPiece<T>::type w;
#pragma unroll
        for (int e = 0; e < 8; e++)
            w[e] = (T)v[e];
        __builtin_nontemporal_store(w, reinterpret_cast<typename RecdPiece<T>::type *>(p));
    }
}
