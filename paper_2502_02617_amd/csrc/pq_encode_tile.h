/*
 * pq_encode_tile.h -- device code shared by the kernels that encode whole tiles: a tile's
 * image and strings in LDS, and the operands of the product with S.
 */
#ifndef PQ_ENCODE_TILE_H
#define PQ_ENCODE_TILE_H

#include "pq_common.h"
#include "pq_polar.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

/* tile image in LDS: the code bytes, then the radius plane (512 binary16 block radii, or at
   depth 7 the 64 words of radius and upper-level codes) */
template <bool DEEP> struct TileImage {
    static constexpr int radii_halves = DEEP ? PQ_DEEP_RADII_HALVES : PQL_RADII;
    static constexpr int dwords = (PQL_CODE_BYTES + radii_halves * 2) / 4; /* 992 or 800 */
};

__device__ __forceinline__ uint32_t bf16_rne_bits(float f)
{
    uint32_t u = __float_as_uint(f);
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

union BOperand {
    bf16x8 v;
    f16x8 h;
    uint4 q;
    uint32_t w[4];
};

/* ---- partially written tiles: an image of the tile's present contents in LDS, into which the fields of block b of slot
 * tau are scattered without branches: every field's bits are cleared and the field, shifted to its place inside a pair of
 * dwords, is OR-ed in.  The image is shared by the lanes of one wavefront and the fields of different slots share
 * dwords: LDS atomics.  The positions are those of pq_layout.h, written out per plane. ---- */
__device__ __forceinline__ void put_pair(uint32_t *img, uint32_t at0, uint32_t at1, uint32_t field, uint32_t width, uint32_t sh)
{
    const uint64_t m = (uint64_t)((1u << width) - 1u) << sh;
    atomicAnd(&img[at0], ~(uint32_t)m);
    atomicAnd(&img[at1], ~(uint32_t)(m >> 32));
    const uint64_t w = (uint64_t)field << sh;
    atomicOr(&img[at0], (uint32_t)w);
    atomicOr(&img[at1], (uint32_t)(w >> 32));
}

template <int KIND, bool DEEP>
__device__ __forceinline__ void emit_block(uint32_t *img, int tau, int b, const BlockCodes &bc)
{
    const uint32_t q0 = bc.q[0], q1 = bc.q[1], q2 = bc.q[2], q3 = bc.q[3], bi = bc.bi;
    uint32_t radius_half;
    if (KIND == PQ_KEY) {
        /* dword d of the token's string: planes of 4, 4, 3 dwords per token, then one half per token */
        auto at = [&](uint32_t d) {
            return d < 4u ? 4u * tau + d : d < 8u ? (PQL_OFF_P1 / 4 - 4) + 4u * tau + d
                 : d < 11u ? (PQL_OFF_P2 / 4 - 8) + 3u * tau + d : PQL_OFF_KP3 / 4 + ((uint32_t)tau >> 1);
        };
        const uint32_t bit = PQL_BLOCK_BITS * (uint32_t)b, d = bit >> 5, sh = bit & 31u;
        /* the string's last half sits in a dword shared by two tokens */
        const uint32_t sh1 = (d + 1u == 11u) ? 16u * ((uint32_t)tau & 1u) : 0u;
        /* 46 bits reach into a third dword when they start above bit 18 (never in the string's last dwords) */
        const bool third = sh > 18u;
        const uint32_t a0 = at(d), a1 = at(d + 1u), a2 = at(third ? d + 2u : d);
        const uint64_t m = ((1ull << PQL_BLOCK_BITS) - 1ull) << sh;
        atomicAnd(&img[a0], ~(uint32_t)m);
        atomicAnd(&img[a1], ~((uint32_t)(m >> 32) << sh1));
        if (third) atomicAnd(&img[a2], ~(0x3FFFu >> (32u - sh)));
        const uint32_t lo = q0 | (q1 << 10) | (q2 << 20) | (q3 << 30), hi = (q3 >> 2) | (bi << 8); /* 32 + 14 bits */
        const uint64_t w = (((uint64_t)hi << 32) | lo) << sh;
        atomicOr(&img[a0], (uint32_t)w);
        atomicOr(&img[a1], (uint32_t)(w >> 32) << sh1);
        if (third) atomicOr(&img[a2], hi >> (32u - sh));
        radius_half = 8u * tau + b;
    } else {
        const uint32_t i = (uint32_t)tau >> 4, g = ((uint32_t)tau >> 2) & 3u, e = (uint32_t)tau & 3u, s = 4u * i + e;
        /* dword d of lane lam's string: planes of 4, 4, 2 dwords per lane */
        auto at = [&](uint32_t lam, uint32_t d) {
            return d < 4u ? 4u * lam + d : d < 8u ? (PQL_OFF_P1 / 4 - 4) + 4u * lam + d : (PQL_OFF_P2 / 4 - 8) + 2u * lam + d;
        };
        const uint32_t bit = PQL_SLOT_BITS * s, d = bit >> 5, sh = bit & 31u;
        /* the dword after a string's last one belongs to the next lane (or the next plane): it gets zeros */
        const uint32_t lam0 = 16u * g + 2u * b;
        put_pair(img, at(lam0, d), at(lam0, d + 1u), q0 | (q1 << 10), PQL_SLOT_BITS, sh);
        put_pair(img, at(lam0 + 1u, d), at(lam0 + 1u, d + 1u), q2 | (q3 << 10), PQL_SLOT_BITS, sh);
        const uint32_t bbit = 6u * s, base = PQL_OFF_VB / 4 + 3u * (8u * g + b) + (bbit >> 5);
        put_pair(img, base, base + 1u, bi, 6u, bbit & 31u);
        radius_half = 16u * (8u * g + b) + s;
    }
    if (!DEEP) reinterpret_cast<uint16_t *>(img)[PQL_CODE_BYTES / 2 + radius_half] = bc.radius;
}

/* ---- whole tiles: every block leaves its indices and radius in LDS at a place of its own (plain writes, compile-time
 * shifts), and once the tile is complete a lane reads the blocks of its strings, joins them and stores
 * full-width dwords.  An image for whole tiles too, with its addresses and atomics, made the keys and values of 32768
 * tokens 64.1 us against 57.6 (235 against 219 at four times as many; one-term S 43.3 against 41.8; value tiles
 * gain most: 34.9 against 30.6 for 262144 vectors, keys 30.7 against 30.2).
 *   keys:   [block][token] of two dwords: Q0 | Q1 << 10 | Q2 << 20 | Q3 << 30, then Q3 >> 2 | B << 8 | radius << 16
 *   values: [half-block][token] of one dword: its two indices, for the first half also B << 20; behind them the
 *           radii [block][token].  Rows of 68 dwords and 68 halves: the reads of 16 half-blocks (8 blocks) at one token
 *           then fall on different banks. ---- */
constexpr int kRow = 68, kRadiiAt = 16 * kRow /* dwords */, kWaveDwords = kRadiiAt + 8 * kRow / 2;

template <int KIND, bool DEEP>
__device__ __forceinline__ void leave_block(uint32_t *buf, int tau, int b, const BlockCodes &bc)
{
    if (KIND == PQ_KEY) {
        const uint32_t lo = bc.q[0] | (bc.q[1] << 10) | (bc.q[2] << 20) | (bc.q[3] << 30);
        uint32_t hi = (bc.q[3] >> 2) | (bc.bi << 8);
        if (!DEEP) hi |= (uint32_t)bc.radius << 16;
        *reinterpret_cast<uint2 *>(buf + 2 * (64 * b + tau)) = make_uint2(lo, hi);
    } else {
        buf[(2 * b) * kRow + tau] = bc.q[0] | (bc.q[1] << 10) | (bc.bi << 20);
        buf[(2 * b + 1) * kRow + tau] = bc.q[2] | (bc.q[3] << 10);
        if (!DEEP) reinterpret_cast<uint16_t *>(buf + kRadiiAt)[b * kRow + tau] = bc.radius;
    }
}

/* `width` bits of v (the others zero) to bit BIT of the string w, whose bits from there on are zero */
template <int BIT, int WIDTH>
__device__ __forceinline__ void put_field(uint32_t *w, uint32_t v)
{
    constexpr int d = BIT >> 5, s = BIT & 31;
    if constexpr (s == 0) w[d] = v;
    else {
        w[d] |= v << s;
        if constexpr (s + WIDTH > 32) w[d + 1] = v >> (32 - s);
    }
}

template <bool DEEP, int B>
__device__ __forceinline__ void join_key_block(uint32_t (&w)[12], uint32_t (&rad)[4], const uint32_t *buf, int lane)
{
    const uint2 f = *reinterpret_cast<const uint2 *>(buf + 2 * (64 * B + lane));
    put_field<PQL_BLOCK_BITS * B, 32>(w, f.x);
    put_field<PQL_BLOCK_BITS * B + 32, 14>(w, DEEP ? f.y : f.y & 0x3FFFu);
    if (!DEEP) rad[B / 2] = (B & 1) ? __builtin_amdgcn_perm(f.y, rad[B / 2], 0x07060100u) : f.y >> 16;
}

template <int I, bool DEEP>
__device__ __forceinline__ void join_value_slots(uint32_t (&w)[10], uint32_t (&vb)[3], uint32_t (&rad)[4], const uint32_t *buf, int lane)
{
    const int g = lane >> 4, n = lane & 15;
    const uint4 f = *reinterpret_cast<const uint4 *>(buf + n * kRow + 16 * I + 4 * g); /* slots 4 I .. 4 I + 3 */
    put_field<PQL_SLOT_BITS * (4 * I), 20>(w, f.x & 0xFFFFFu);
    put_field<PQL_SLOT_BITS * (4 * I + 1), 20>(w, f.y & 0xFFFFFu);
    put_field<PQL_SLOT_BITS * (4 * I + 2), 20>(w, f.z & 0xFFFFFu);
    put_field<PQL_SLOT_BITS * (4 * I + 3), 20>(w, f.w & 0xFFFFFu);
    put_field<6 * (4 * I), 6>(vb, f.x >> 20);
    put_field<6 * (4 * I + 1), 6>(vb, f.y >> 20);
    put_field<6 * (4 * I + 2), 6>(vb, f.z >> 20);
    put_field<6 * (4 * I + 3), 6>(vb, f.w >> 20);
    if (!DEEP && I < 2) { /* half n & 1 of the block stores slots 8 (n & 1) .. + 7 of its radii */
        const uint2 r = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(buf + kRadiiAt) + (n >> 1) * kRow +
                                                         16 * (2 * (n & 1) + I) + 4 * g);
        rad[2 * I] = r.x;
        rad[2 * I + 1] = r.y;
    }
}

/* the strings and radii of a whole tile, one lane per token (keys) or half-block of 16 tokens (values) */
template <int KIND, bool DEEP>
__device__ __forceinline__ void store_tile(const uint32_t *buf, uint8_t *gcodes, uint16_t *gradii, int lane)
{
    struct Three { uint32_t x, y, z; };
    uint32_t rad[4];
    if (KIND == PQ_KEY) {
        uint32_t w[12];
        join_key_block<DEEP, 0>(w, rad, buf, lane); join_key_block<DEEP, 1>(w, rad, buf, lane);
        join_key_block<DEEP, 2>(w, rad, buf, lane); join_key_block<DEEP, 3>(w, rad, buf, lane);
        join_key_block<DEEP, 4>(w, rad, buf, lane); join_key_block<DEEP, 5>(w, rad, buf, lane);
        join_key_block<DEEP, 6>(w, rad, buf, lane); join_key_block<DEEP, 7>(w, rad, buf, lane);
        reinterpret_cast<uint4 *>(gcodes + PQL_OFF_P0)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(gcodes + PQL_OFF_P1)[lane] = make_uint4(w[4], w[5], w[6], w[7]);
        reinterpret_cast<Three *>(gcodes + PQL_OFF_P2)[lane] = Three{w[8], w[9], w[10]};
        reinterpret_cast<uint16_t *>(gcodes + PQL_OFF_KP3)[lane] = (uint16_t)w[11];
    } else {
        uint32_t w[10], vb[3];
        join_value_slots<0, DEEP>(w, vb, rad, buf, lane); join_value_slots<1, DEEP>(w, vb, rad, buf, lane);
        join_value_slots<2, DEEP>(w, vb, rad, buf, lane); join_value_slots<3, DEEP>(w, vb, rad, buf, lane);
        reinterpret_cast<uint4 *>(gcodes + PQL_OFF_P0)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(gcodes + PQL_OFF_P1)[lane] = make_uint4(w[4], w[5], w[6], w[7]);
        reinterpret_cast<uint2 *>(gcodes + PQL_OFF_P2)[lane] = make_uint2(w[8], w[9]);
        if ((lane & 1) == 0) reinterpret_cast<Three *>(gcodes + PQL_OFF_VB)[lane >> 1] = Three{vb[0], vb[1], vb[2]};
    }
    if (!DEEP) reinterpret_cast<uint4 *>(gradii)[lane] = make_uint4(rad[0], rad[1], rad[2], rad[3]);
}

/* lanes 0..31: the value of lane + 32; lanes 32..63: the value of lane - 32 */
__device__ __forceinline__ uint32_t from_other_half(uint32_t x, int upper_half)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return upper_half ? r[0] : r[1];
}

/* NTERMS = 3: S as three bf16 terms.  NTERMS = 1: every entry of S is +-1/sqrt(128), the
   operand is sqrt(128) * S (exactly +-1), one product per k-step replaces three and
   the common factor is taken out of the block radius (the angles do not see it).
   NTERMS = 2: S as two binary16 terms of 2^15 S, 23 significant bits.

   fp32 input with NTERMS = 1 or 2 is two binary16 terms as well, after a power of two has brought the vector's
   largest coordinate to [2^14, 2^15) (the factor comes out of the radius, the angles do not see it): three products
   (two for a +-1 S) instead of the six (three) that three bf16 terms of 8 bits take, and a third of the vector
   instructions to split an input: keys and values of 32768 tokens of 8 heads 116 -> 82 us, 89 -> 72 with a +-1 S.
   Operands: two terms leave up to 2^-23 of a number (three bf16 terms 2^-25), or 2^-39 of the vector's largest coordinate where that
   is more, and the product that is left out is 2^-22 of its whole at most; rms 7e-8 of a product, ten times that of three bf16 terms.
   The fp32 sums, which are half as many, round by more: of 268 M radii of vectors with outlier channels 7.2e-5 differ by a last
   bit from 64 bits (three bf16 terms 8.0e-5), of coordinates spread over 2^12 4.7e-5 (5.1e-5); with a Hadamard S, whose entries
   are exact, 7.0e-5 (7.2e-5) and, spread, 4.68e-5 (4.53e-5: there it is larger, by 3 %).
   2^-39 of the largest coordinate per coordinate is 2^-40 of it rms in a rotated one (the columns of S have norm 1).  Sums that pass
   2^-16 of it round by 2^-41 rms at each of the products behind, a dozen on average of 24: 2^-39.  So an S that
   spreads every coordinate over all pairs of the result by 2^-16 at least (pq_ctx::mixing) does not see it; any other keeps
   NTERMS = 3. */
template <int XT, int NTERMS> struct Operands {
    static constexpr bool half = XT == PQ_F32 && NTERMS <= 2;             /* binary16 terms, else bf16 */
    static constexpr int x_terms = XT == PQ_BF16 ? 1 : (half ? 2 : 3);
    static constexpr int top = NTERMS == 3 ? 2 : 1;                       /* products of terms x + s <= top take part */
    static constexpr int products = x_terms == 1 ? NTERMS : (NTERMS == 3 ? 6 : NTERMS + 1); /* of a k-step */
    static constexpr int s_chunks = NTERMS * 4 * 8 * 64;                  /* 16-byte chunks of S in LDS */
};

template <int XT, int NTERMS>
__device__ __forceinline__ f32x16 multiply(const BOperand &s, const BOperand &x, const f32x16 &c)
{
    if constexpr (Operands<XT, NTERMS>::half) return __builtin_amdgcn_mfma_f32_32x32x16_f16(s.h, x.h, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(s.v, x.v, c, 0, 0, 0);
}

/* Chunk of S as the matrix instructions take it, from the chunks of its bf16 terms (t[1], t[2]: NTERMS > 1). */
template <int XT, int NTERMS>
__device__ __forceinline__ void s_operand(BOperand (&out)[NTERMS], const uint4 *t)
{
    if constexpr (NTERMS == 2) {
        BOperand b[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) b[k].q = t[k];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float f[3];
#pragma unroll
            for (int k = 0; k < 3; ++k)
                f[k] = 32768.f * __uint_as_float((e & 1) ? b[k].w[e / 2] & 0xFFFF0000u : b[k].w[e / 2] << 16);
            const _Float16 hi = (_Float16)(f[0] + f[1]);
            out[0].h[e] = hi;
            out[1].h[e] = (_Float16)((f[0] - (float)hi) + f[1] + f[2]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < NTERMS; ++k) out[k].q = t[k];
        if constexpr (Operands<XT, NTERMS>::half) { /* +-1 */
#pragma unroll
            for (int k = 0; k < 4; ++k) out[0].w[k] = (out[0].w[k] & 0x80008000u) | 0x3C003C00u;
        }
    }
}

/* Eight coordinates as three bf16 terms. */
__device__ __forceinline__ void split_bf16(const float (&f)[8], BOperand (&out)[3])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        uint32_t b[3][2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            float rest = f[e + z];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                b[k][z] = bf16_rne_bits(rest);
                rest -= __uint_as_float(b[k][z] << 16);
            }
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) out[k].w[e / 2] = b[k][0] | (b[k][1] << 16);
    }
}

/* The power of two that brings a vector with largest coordinate m to [2^14, 2^15), as a biased exponent: at least 13 (an
   infinity among the inputs), and 2^103 at most. */
__device__ __forceinline__ uint32_t half_exponent(float m) { return min(268u - (__float_as_uint(m) >> 23), 230u); }

/* What the rotated coordinates have to be multiplied with: the power of two and, with two terms of S, its 2^15. */
template <int NTERMS>
__device__ __forceinline__ float half_unscale(uint32_t e) { return __uint_as_float(((NTERMS == 1 ? 254u : 239u) - e) << 23); }

/* Eight coordinates times the power of two of exponent e as two binary16 terms. */
__device__ __forceinline__ void split_half(const float (&f)[8], uint32_t e, BOperand (&out)[2])
{
    const float scale = __uint_as_float(e << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const _Float16 hi = (_Float16)(f[i] * scale);
        out[0].h[i] = hi;
        out[1].h[i] = (_Float16)__builtin_fmaf(f[i], scale, -(float)hi);
    }
}

__device__ __forceinline__ float max_abs(float m, const float4 &a)
{
    return fmaxf(fmaxf(m, fmaxf(fabsf(a.x), fabsf(a.y))), fmaxf(fabsf(a.z), fabsf(a.w)));
}

} // namespace

#endif /* PQ_ENCODE_TILE_H */
