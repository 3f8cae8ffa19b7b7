/*
 * pq_paged.hip -- pq_append_paged: the keys and values of a ragged batch of new tokens to a paged cache, with the
 * position rotation of the keys on the way (Algorithm 1 lines 2 and 4 on k' = Rot(position) k and on v).
 *
 * Codes are settled in double precision: y = k' S with S, the rotation's products and the sums in 64 bits, and the
 * cell comparisons v > tan(t) u of procedure Quant as well (their squares above level 1).  A vector therefore gets
 * the codes of the definition whatever batch it comes in, and equal prefixes have equal pages.
 */
#include <type_traits>

#include "pq_common.h"
#include "pq_encode_tile.h"
#include "pq_paged.h"
#include "pq_polar.h"

namespace {

struct AppendPagedArgs {
    const void *x[2]; /* keys, values */
    uint8_t *codes[2];
    uint16_t *radii[2];
    int64_t ld_token, ld_head;
    int n_heads;
    PagedTable table;
    PagedRows rows;
    RotaryArgs rot;
    const int32_t *positions;
    const PqExact *exact;
    const PqDeviceConsts *consts;
};

/* A row of the batch: its sequence's token, and where that lies in the pool (page -1: nowhere, nothing is written). */
struct PagedPlace {
    int64_t page, position;
    int tau;
};

__device__ __forceinline__ PagedPlace paged_place(const AppendPagedArgs &a, int64_t row, int lane)
{
    PagedPlace p{-1, 0, 0};
    const int b = paged_find(a.rows.n_seq, row, lane, [&](int i) { return (int64_t)a.rows.row_start[i]; });
    if (b < 0 || b >= a.rows.n_seq) return p;
    const int64_t token = (int64_t)a.rows.ctx_len[b] - (a.rows.row_start[b + 1] - row);
    p.page = paged_page(a.table, b, token);
    p.tau = (int)(token & 63);
    p.position = a.positions ? (int64_t)a.positions[row] : token;
    return p;
}

/* The boundaries that settle codes, requested ahead of the vector they are for. */
struct ExactBounds {
    double tan1[3], tan2[3][3];
    bool general, deep;
    __device__ __forceinline__ void load(const PqExact &E, const PqDeviceConsts &K)
    {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            tan1[k] = E.tan1[k];
#pragma unroll
            for (int l = 0; l < 3; ++l) tan2[l][k] = E.tan2[l][k];
        }
        general = K.general != 0;
        deep = K.depth == 7;
    }
};

/* procedure Quant inside a quadrant, in 64 bits: boundaries below atan(v / u), u, v >= 0 (or of squares, with squared tangents) */
__device__ __forceinline__ uint32_t quant3_exact(double u, double v, const double (&t)[3])
{
    return (v > t[0] * u ? 1u : 0u) + (v > t[1] * u ? 1u : 0u) + (v > t[2] * u ? 1u : 0u);
}

__device__ __forceinline__ uint32_t quant_upper_exact(double u2, double v2, const double *tan2, int n_bounds)
{
    uint32_t c = 0;
    for (int k = 0; k < n_bounds; ++k) c += v2 > tan2[k] * u2 ? 1u : 0u;
    return c;
}

/* level-1 code of (ya, yb): quadrant from the signs and the cell inside it, or the number of boundaries below its pseudo-angle */
__device__ __forceinline__ uint32_t level1_exact(double ya, double yb, const PqExact &E, const ExactBounds &B)
{
    const uint32_t sa = (uint32_t)(__double2hiint(ya)) >> 31, sb = (uint32_t)(__double2hiint(yb)) >> 31, f = sa ^ sb;
    const double a = fabs(ya), b = fabs(yb);
    if (!B.general) return (quant3_exact(a, b, B.tan1) ^ (f ? 7u : 0u)) | (sb << 3);
    const double sum = a + b;
    const double p = (double)(2u * sb + f) + (sum > 0.0 ? (f ? a : b) / sum : 0.0);
    uint32_t c = 0;
    for (int k = 0; k < 15; ++k) c += p > E.pseudo1[k] ? 1u : 0u;
    return c;
}

/* one rounding, to nearest even */
__device__ __forceinline__ uint16_t radius_exact(double q)
{
    return __builtin_bit_cast(uint16_t, (_Float16)fmin(sqrt(q), 65504.0));
}

/* x of the lane that the DPP control names, inside rows of sixteen lanes */
template <int CTRL>
__device__ __forceinline__ double dpp_double(double x)
{
    return __hiloint2double(pq_dpp<CTRL>(__double2hiint(x)), pq_dpp<CTRL>(__double2loint(x)));
}

__device__ __forceinline__ double shfl_xor_double(double x, int d)
{
    const int lo = __shfl_xor(__double2loint(x), d), hi = __shfl_xor(__double2hiint(x), d);
    return __hiloint2double(hi, lo);
}

/* One rotated vector, coordinates 2 p and 2 p + 1 in lane p, to slot tau of a page: the recursion of procedure Polar with the codes'
 * comparisons, the nodes above level 1 in the lanes of their first leaf (the others compute the same along). */
template <int KIND>
__device__ __forceinline__ void write_exact(const AppendPagedArgs &a, const ExactBounds &B, double ya, double yb, int64_t tile, int tau, int lane)
{
    const PqExact &E = *a.exact;
    const PqDeviceConsts &K = *a.consts;
    const int i = lane & 7, b = lane >> 3;
    const uint32_t code1 = level1_exact(ya, yb, E, B);
    const double q1 = ya * ya + yb * yb, q1s = dpp_double<0xB1>(q1); /* lane ^ 1 */
    const uint32_t c2 = quant3_exact(q1, q1s, B.tan2[0]);
    const double q2 = q1 + q1s, q2s = dpp_double<0x4E>(q2); /* lane ^ 2 */
    const uint32_t c3 = quant3_exact(q2, q2s, B.tan2[1]);
    const double q3 = q2 + q2s, q3s = dpp_double<0x141>(q3); /* lane 7 - i of eight: any lane of the other quad */
    PqBlockFields f;
    f.c4 = quant3_exact(q3, q3s, B.tan2[2]);
    const double q4 = q3 + q3s;
    f.radius = radius_exact(q4);
    /* level-1 codes at their nibbles; [c2(2h) | c3(h) | c2(2h+1)] of half-block h at bits [8 h, 8 h + 6) */
    uint32_t l1 = code1 << (4 * i);
    uint32_t gw = (i & 1) ? 0u : ((i & 2) ? c2 : ((c2 << 4) | (c3 << 2))) << (2 * (i & 4));
    l1 |= pq_dpp<0xB1>(l1); gw |= pq_dpp<0xB1>(gw);
    l1 |= pq_dpp<0x4E>(l1); gw |= pq_dpp<0x4E>(gw);
    l1 |= pq_dpp<0x141>(l1); gw |= pq_dpp<0x141>(gw);
    f.l1 = l1;
    f.g6[0] = gw & 63u;
    f.g6[1] = (gw >> 8) & 63u;
    if (i == 0) {
        pql_put_block<true>(reinterpret_cast<uint32_t *>(a.codes[KIND] + tile * PQL_CODE_BYTES), KIND, tau, b, f);
        if (!B.deep) a.radii[KIND][tile * PQL_RADII + pql_pos(KIND, tau, b).radius_half] = f.radius;
    }
    if (B.deep) { /* levels 5, 6, 7 over the block radii, and the vector's word of the radius plane */
        const int b5 = K.up_bits[0], b6 = K.up_bits[1], b7 = K.up_bits[2];
        const double q4s = shfl_xor_double(q4, 8), q5 = q4 + q4s;
        const uint32_t c5 = quant_upper_exact(q4, q4s, E.up_tan2[0], (1 << b5) - 1);
        const double q5s = shfl_xor_double(q5, 16), q6 = q5 + q5s;
        const uint32_t c6 = quant_upper_exact(q5, q5s, E.up_tan2[1], (1 << b6) - 1);
        const double q6s = shfl_xor_double(q6, 32);
        const uint32_t c7 = quant_upper_exact(q6, q6s, E.up_tan2[2], (1 << b7) - 1);
        uint32_t word = 0;
        for (int j = 0; j < 4; ++j) word |= (uint32_t)__shfl((int)c5, 16 * j) << (j * b5);
        for (int j = 0; j < 2; ++j) word |= (uint32_t)__shfl((int)c6, 32 * j) << (4 * b5 + j * b6);
        word |= (uint32_t)__shfl((int)c7, 0) << (4 * b5 + 2 * b6);
        word |= (uint32_t)radius_exact(q6 + q6s) << 16;
        if (lane == 0) reinterpret_cast<uint32_t *>(a.radii[KIND])[tile * (PQ_DEEP_RADII_HALVES / 2) + tau] = word;
    }
}

/* y = x S of up to NV vectors by 512 threads in 64 bits: thread (kq, j) sums a quarter of the products of column j.  S is fetched once for
 * the NV products (128 KB, what bounds a launch of few vectors); the thread's part is requested first, ahead of the vectors. */
struct ExactSlice {
    double m[32];
    __device__ __forceinline__ void load(const double *S, int tid)
    {
        const int kq = tid >> 7, j = tid & 127;
#pragma unroll
        for (int k = 0; k < 32; ++k) m[k] = S[(32 * kq + k) * PQ_D + j];
    }
};

template <int NV>
struct ExactLds {
    __attribute__((aligned(16))) double x[NV][PQ_D];
    double part[NV][4][PQ_D];
};

template <int NV, typename Lds>
__device__ __forceinline__ void multiply_exact(const ExactSlice &s, Lds &lds, int tid)
{
    const int kq = tid >> 7, j = tid & 127;
    double acc[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) acc[v] = 0.0;
#pragma unroll
    for (int k = 0; k < 32; k += 2)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const double2 x = *reinterpret_cast<const double2 *>(&lds.x[v][32 * kq + k]);
            acc[v] = fma(x.x, s.m[k], acc[v]);
            acc[v] = fma(x.y, s.m[k + 1], acc[v]);
        }
#pragma unroll
    for (int v = 0; v < NV; ++v) lds.part[v][kq][j] = acc[v];
}

template <typename Lds>
__device__ __forceinline__ double rotated_exact(const Lds &lds, int r, int c)
{
    return ((lds.part[r][0][c] + lds.part[r][1][c]) + lds.part[r][2][c]) + lds.part[r][3][c];
}

/* coordinate c of a vector, a key's rotated to its position */
template <int XT>
__device__ __forceinline__ double element_exact(const AppendPagedArgs &a, int kind, int64_t off, int64_t position, int c)
{
    auto element = [&](int k) -> double {
        if (XT == PQ_BF16) return (double)__uint_as_float((uint32_t) static_cast<const uint16_t *>(a.x[kind])[off + k] << 16);
        return (double)static_cast<const float *>(a.x[kind])[off + k];
    };
    double x = element(c);
    if (kind == PQ_KEY && c < a.rot.dim) {
        const RotaryPair p = rotary_pair(a.rot, c);
        const float *cs = rotary_row(a.rot, position);
        const double s = (double)cs[(a.rot.dim >> 1) + p.at] * element(p.partner);
        x = x * (double)cs[p.at] + (p.minus ? -s : s);
    }
    return x;
}

/* Vectors (row, head) of kind KIND, NV at a time, from NV * block on, with NV 8 in steps of 8 * n_blocks: S is fetched once for them all.  Two wavefronts
 * fetch a vector (NV 8: one), the first of them runs its recursion. */
template <int XT, int KIND, int NV>
__device__ __forceinline__ void append_vectors_exact(const AppendPagedArgs &a, int block, int n_blocks, int64_t n_vec, ExactLds<NV> &lds)
{
    constexpr int kWaves = NV == 8 ? 1 : 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    ExactSlice s;
    s.load(a.exact->S, tid);
    ExactBounds bounds;
    bounds.load(*a.exact, *a.consts);
    const int r = min(wave / kWaves, NV - 1); /* a vector beyond the range repeats the last one and is not written */
    const bool mine = wave / kWaves < NV;
    for (int64_t vec0 = (int64_t)NV * block; vec0 < n_vec; vec0 += (int64_t)NV * n_blocks) {
        const int64_t vec = min(vec0 + r, n_vec - 1), row = vec / a.n_heads;
        const int head = (int)(vec - row * a.n_heads);
        int l = lane; /* what follows from the lane is formed here: kept over the loop it takes the second workgroup's registers */
        asm volatile("" : "+v"(l));
        const PagedPlace at = paged_place(a, row, l);
        if (mine) {
            const int64_t off = row * a.ld_token + (int64_t)head * a.ld_head;
#pragma unroll
            for (int i = 0; i < 2 / kWaves; ++i) {
                const int c = l + 64 * (kWaves == 1 ? i : wave & 1);
                lds.x[r][c] = element_exact<XT>(a, KIND, off, at.position, c);
            }
        }
        __syncthreads();
        multiply_exact<NV>(s, lds, tid);
        __syncthreads();
        if (wave % kWaves == 0 && mine && vec0 + r < n_vec && at.page >= 0)
            write_exact<KIND>(a, bounds, rotated_exact(lds, r, 2 * l), rotated_exact(lds, r, 2 * l + 1), head * a.table.pool_pages + at.page, at.tau, l);
        if (NV < 8) return; /* a workgroup for every NV of them */
        /* the next vectors' coordinates go where nobody reads any more, their products behind the next barrier */
    }
}

/* workgroups [0, n_blocks): keys, the rest: values */
template <int XT, int NV>
__global__ __launch_bounds__(512, NV == 8 ? 4 : 1) void pq_append_paged_kernel(AppendPagedArgs a, int64_t n_vec, int n_blocks)
{
    __shared__ ExactLds<NV> lds;
    const int blk = (int)blockIdx.x;
    if (blk < n_blocks) append_vectors_exact<XT, PQ_KEY, NV>(a, blk, n_blocks, n_vec, lds);
    else append_vectors_exact<XT, PQ_VALUE, NV>(a, blk - n_blocks, n_blocks, n_vec, lds);
}

/* ---- whole tiles: chunks of prompts ----
 * A workgroup per tile, as for short inputs of pq_encode_kv: rows are rotated in fp32 and left in LDS as matrix operands, eight threads
 * per vector; wavefront (v, rt) multiplies the 32 vectors of half v into row tile rt of S and runs the recursion of blocks rt and 4 + rt.
 *
 * Codes in doubt.  A rotated coordinate is off by less than E = 2^-23 |x|: 24 products of matrix instructions add to one fp32 sum, whose
 * roundings are 2^-24 of partial sums far below |x|; with 2^-24 in place of 2^-23 no code of 2 * 10^9 was wrong, with 2^-26 13 were, and
 * without any doubt 326.  The code of a node is certain if its inputs u, v are further from every boundary t than that moves the
 * comparison: |tan t u - v| > (1 + tan t) E at level 1, where a coordinate's sign is a boundary as well; above it, where squares are
 * compared, |tan^2 t u^2 - v^2| > 2 sqrt 2 E |(u, v)| sin t (1 + tan t).  The largest factor of a level's boundaries serves for all, and
 * |(u, v)| is bounded from above by (q / s + s) / 2, q = u^2 + v^2, with s the node's usual radius: doubt is only ever found too often, in 1 of
 * 500 vectors without a preferred direction.  The workgroup lists them and, behind its last tile, codes them once more in 64 bits, eight at a
 * time, a wavefront each (5 us; four at a time, twice as many in doubt: 8192 tokens of 8 heads 46 us, now 41). */
constexpr float kDoubt = 0x1p-23f;
constexpr int kChunkItems = 256; /* tiles of one workgroup at most */
constexpr int kListed = 256;     /* vectors that are coded once more in one go */

struct ChunkItem { /* a tile that the workgroup has written */
    int32_t page, row0, token0, head_kind;
};

/* what the certainty of a vector's codes is measured with */
struct Doubt {
    float e;          /* level 1: (1 + tan 3 pi / 8) E */
    float b2, b3, b4; /* the vector's part of the bounds of levels 2, 3, 4 */
};

/* What a level's bound is made of: 2 sqrt 2 E f (q / s + s) / 2 = c q + b |x|^2 with s = rho |x|, a node's radius among 128 coordinates, f the
   level's factor (PqExact::doubt); and 2^-21 q for the roundings of the squares and their sums. */
struct DoubtLevels {
    float c2, c3, c4, b2, b3, b4;
};

__device__ __forceinline__ DoubtLevels doubt_levels(const PqExact &E)
{
    constexpr float kRho2 = 0.1767767f, kRho3 = 0.25f, kRho4 = 0.3535534f, k = 1.4142136f * kDoubt;
    return DoubtLevels{__builtin_fmaf(E.doubt[0], k / kRho2, 0x1p-21f), __builtin_fmaf(E.doubt[1], k / kRho3, 0x1p-21f),
                       __builtin_fmaf(E.doubt[2], k / kRho4, 0x1p-21f), E.doubt[0] * (k * kRho2), E.doubt[1] * (k * kRho3), E.doubt[2] * (k * kRho4)};
}

__device__ __forceinline__ Doubt doubt_of(float norm2, const DoubtLevels &l)
{
    return Doubt{3.4142136f * kDoubt * __builtin_amdgcn_sqrtf(norm2), norm2 * l.b2, norm2 * l.b3, norm2 * l.b4};
}

__device__ __forceinline__ float min3_abs(float a, float b, float c) { return fminf(fminf(fabsf(a), fabsf(b)), fabsf(c)); }

/* distance of a node above level 1 from its nearest boundary, less the node's part of what it may be off */
__device__ __forceinline__ float doubt_node(float u, float v, float t1, float t2, float t3, float c)
{
    return __builtin_fmaf(-c, u + v, min3_abs(__builtin_fmaf(t1, u, -v), __builtin_fmaf(t2, u, -v), __builtin_fmaf(t3, u, -v)));
}

/* polar_quant_block, and whether a code is in doubt */
template <bool GENERAL>
__device__ __forceinline__ BlockCodes quant_block_checked(const f32x16 &y, const Thresholds &th, const Doubt &d, const DoubtLevels &l, const float *pseudo,
                                                          bool &doubt)
{
    PolarState s;
    float near1 = INFINITY, near2 = INFINITY, near3 = INFINITY;
    const float t2b = GENERAL ? th.t2b : 1.f, t3b = GENERAL ? th.t3b : 1.f, t4b = GENERAL ? th.t4b : 1.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        polar_level1_a<GENERAL>(s, y, p, th);
        const float a = fabsf(y[2 * p]), b = fabsf(y[2 * p + 1]);
        if (GENERAL) {
            /* pseudo-angle: off by 2 E / (a + b) and a rounding of numbers below 4 */
            const float sum = a + b;
            const uint32_t ba = __float_as_uint(y[2 * p]), bb = __float_as_uint(y[2 * p + 1]), sb = bb >> 31, f = (ba ^ bb) >> 31;
            const float pa = (float)(2u * sb + f) + (sum > 0.f ? (f ? a : b) * __builtin_amdgcn_rcpf(sum) : 0.f);
            const float gap = fminf(pa - pseudo[s.mq], pseudo[s.mq + 1] - pa);
            near1 = fminf(near1, (gap - 0x1p-20f) * sum);
        } else {
            near1 = fminf(fminf(near1, fminf(a, b)), min3_abs(__builtin_fmaf(th.t1a, a, -b), a - b, __builtin_fmaf(th.t1c, a, -b)));
        }
        polar_level1_b<GENERAL>(s, y, p);
        polar_upper<GENERAL>(s, p, th);
        if (p & 1) {
            const int n = p >> 1;
            near2 = fminf(near2, doubt_node(s.q1[2 * n], s.q1[2 * n + 1], th.t2a, t2b, th.t2c, l.c2));
        }
        if ((p & 3) == 3) {
            const int h = p >> 2;
            near3 = fminf(near3, doubt_node(s.q2[2 * h], s.q2[2 * h + 1], th.t3a, t3b, th.t3c, l.c3));
        }
    }
    const float near4 = doubt_node(s.q3[0], s.q3[1], th.t4a, t4b, th.t4c, l.c4);
    doubt = near1 < d.e || near2 < d.b2 || near3 < d.b3 || near4 < d.b4;
    return s.out;
}

/* the same of a node of levels 5, 6, 7 */
__device__ __forceinline__ bool upper_in_doubt(float u2, float v2, const float *tan2, float factor, int n_bounds, float e)
{
    const float q = u2 + v2, bound = 2.8284271f * factor * e * __builtin_amdgcn_sqrtf(q) + 0x1p-20f * q;
    bool doubt = false;
#pragma unroll
    for (int k = 0; k < 7; ++k)
        if (k < n_bounds) doubt |= fabsf(__builtin_fmaf(tan2[k], u2, -v2)) < bound;
    return doubt;
}

/* maximum and sum over the eight lanes lane & 7 + 8 k */
__device__ __forceinline__ float over_parts_max(float x)
{
    x = fmaxf(x, pq_dpp<0x128>(x)); /* row_ror:8 */
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

__device__ __forceinline__ float over_parts_sum(float x)
{
    x += pq_dpp<0x128>(x);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

template <int XT, int NTERMS, bool GENERAL, bool DEEP>
__global__ __launch_bounds__(512) void pq_append_chunk_kernel(AppendPagedArgs a, const uint4 *S_terms, int64_t n_items)
{
    typedef Operands<PQ_F32, NTERMS> Op; /* rotated rows are fp32, whatever the input's type */
    constexpr int NXT = Op::x_terms, kThreads = 512;
    constexpr int kImgDwords = TileImage<DEEP>::dwords, kRadiiHalves = TileImage<DEEP>::radii_halves;
    constexpr int kRows = NXT * 8 * 2 * 64; /* a tile's rows, [term][k-step][half][lane] */
    constexpr int kRaw = XT == PQ_BF16 ? 2 : 4;
    __shared__ union {
        uint4 rows[2 * kRows];
        ExactLds<8> exact;
    } lds;
    __shared__ __align__(16) uint32_t sImg[2][kWaveDwords];
    __shared__ float sQ4[DEEP ? 2 : 1][2][4][DEEP ? 64 : 1];
    __shared__ float sUnscale[2][64], sNorm2[2][64];
    __shared__ PqDeviceConsts::Lut1Cell sLut[GENERAL ? 512 : 1];
    __shared__ float sPseudo[17];
    __shared__ ChunkItem sItem[kChunkItems];
    __shared__ uint32_t sDoubt[kChunkItems][2];
    __shared__ uint32_t sList[kListed];
    __shared__ int sCount;
    /* the rotation table's rows of a tile's tokens: a tile's heads follow each other.  Rows of 132: the eight vectors of a wavefront then
       begin on different banks. */
    __shared__ __align__(16) float sTurn[64][132];
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, H = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), v = wave & 1, rt = wave >> 1;
    /* items: tile numbers, for each the keys of all heads, then the values: a workgroup has consecutive ones, so a tile's place is looked
       up once for many of them and its rotation table's rows stay near */
    const int per_tile = 2 * a.n_heads;
    struct Item {
        int u, rest;                /* tile number, item of the tile */
        int page, row0, lo, hi;     /* slots [lo, hi) are written, slot tau from row row0 + tau */
        int token0;
        int some;                   /* 0: behind the last (an int: the padding behind a bool is copied through memory) */
    };
    const int64_t first_item = (int64_t)blockIdx.x * n_items / gridDim.x, item_end = (int64_t)(blockIdx.x + 1) * n_items / gridDim.x;
    const int u_end = (int)(item_end / per_tile), rest_end = (int)(item_end % per_tile);
    auto look_up = [&](Item &it) { /* from item (u, rest) on, the next one that has something to write */
        for (;;) {
            it.some = it.u < u_end || (it.u == u_end && it.rest < rest_end);
            if (!it.some) return;
            const PagedTile t = paged_tile(a.table, a.rows, it.u, lane);
            if (t.page >= 0 && t.lo < t.hi) {
                it.page = (int)t.page;
                it.row0 = (int)t.row0;
                it.lo = (int)max(t.lo - t.row0, (int64_t)0);
                it.hi = (int)min(t.hi - t.row0, (int64_t)64);
                it.token0 = (int)t.token0;
                return;
            }
            ++it.u;
            it.rest = 0;
        }
    };
    auto following = [&](const Item &from) {
        Item it = from;
        if (++it.rest == per_tile) {
            it.rest = 0;
            ++it.u;
            look_up(it);
        } else {
            it.some = it.u < u_end || (it.u == u_end && it.rest < rest_end);
        }
        return it;
    };
    auto kind_of = [&](const Item &it) { return it.rest >= a.n_heads ? PQ_VALUE : PQ_KEY; };
    auto head_of = [&](const Item &it) { return it.rest >= a.n_heads ? it.rest - a.n_heads : it.rest; };

    /* this thread's sixteen coordinates 16 part .. + 15 of vector vec, in two pieces of eight; a slot that is not written gets the first row
       that is */
    const int vec = 8 * wave + (lane & 7), part = lane >> 3, half_dim = a.rot.dim >> 1;
    uint4 raw[kRaw], other[kRaw];
    auto load_row = [&](const Item &it) {
        const int kind = kind_of(it);
        const int64_t row = it.row0 + (vec >= it.lo && vec < it.hi ? vec : it.lo), off = row * a.ld_token + (int64_t)head_of(it) * a.ld_head;
        constexpr int kBytes = XT == PQ_BF16 ? 2 : 4;
        const char *base = static_cast<const char *>(a.x[kind]) + off * kBytes;
#pragma unroll
        for (int k = 0; k < kRaw; ++k) raw[k] = reinterpret_cast<const uint4 *>(base + 16 * part * kBytes)[k];
        if (kind != PQ_KEY || 16 * part >= a.rot.dim || a.rot.interleaved) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) { /* dim is a multiple of 16, its half one of 8: a piece lies in one half of the pairs */
            const int c = 16 * part + 8 * k, partner = c < half_dim ? c + half_dim : c - half_dim;
#pragma unroll
            for (int q = 0; q < kRaw / 2; ++q) other[(kRaw / 2) * k + q] = reinterpret_cast<const uint4 *>(base + partner * kBytes)[q];
        }
    };
    int turn_of = -1; /* the tile whose rows are in sTurn */
    auto needs_turn = [&](const Item &it) { return a.rot.cs && it.some && kind_of(it) == PQ_KEY && it.u != turn_of; };
    auto load_turn = [&](const Item &it) { /* all threads, and a barrier before and behind */
        const int at = tid >> 3, slot = at >= it.lo && at < it.hi ? at : it.lo;
        const float *cs = rotary_row(a.rot, a.positions ? (int64_t)a.positions[it.row0 + slot] : (int64_t)it.token0 + slot);
        float4 t[4]; /* all requested before the first is stored; columns from dim on are nobody's */
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = *reinterpret_cast<const float4 *>(cs + min(4 * (tid & 7) + 32 * k, a.rot.dim - 4));
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<float4 *>(&sTurn[at][4 * (tid & 7) + 32 * k]) = t[k];
        turn_of = it.u;
    };
    auto floats = [](const uint4 *r, float (&f)[8]) {
        if constexpr (XT == PQ_BF16) {
            const uint32_t w[4] = {r[0].x, r[0].y, r[0].z, r[0].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float((e & 1) ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        } else {
            const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
        }
    };
    auto leave_row = [&](int buffer, int kind) {
        float f[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            floats(raw + (kRaw / 2) * k, f[k]);
            const int c = 16 * part + 8 * k;
            if (kind == PQ_KEY && c < a.rot.dim) {
                const float *cs = &sTurn[vec][a.rot.interleaved ? c / 2 : (c < half_dim ? c : c - half_dim)];
                const float4 c0 = *reinterpret_cast<const float4 *>(cs), s0 = *reinterpret_cast<const float4 *>(cs + half_dim);
                const float cc[4] = {c0.x, c0.y, c0.z, c0.w}, ss[4] = {s0.x, s0.y, s0.z, s0.w};
                if (a.rot.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = f[k][2 * e], y = f[k][2 * e + 1];
                        f[k][2 * e] = __builtin_fmaf(x, cc[e], -(y * ss[e]));
                        f[k][2 * e + 1] = __builtin_fmaf(x, ss[e], y * cc[e]);
                    }
                } else {
                    const float4 c1 = *reinterpret_cast<const float4 *>(cs + 4), s1 = *reinterpret_cast<const float4 *>(cs + half_dim + 4);
                    const float dd[4] = {c1.x, c1.y, c1.z, c1.w}, tt[4] = {s1.x, s1.y, s1.z, s1.w};
                    float o[8];
                    floats(other + (kRaw / 2) * k, o);
                    const float sign = c < half_dim ? -1.f : 1.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        f[k][e] = __builtin_fmaf(f[k][e], cc[e], sign * (o[e] * ss[e]));
                        f[k][4 + e] = __builtin_fmaf(f[k][4 + e], dd[e], sign * (o[4 + e] * tt[e]));
                    }
                }
            }
        }
        /* k-steps 2 (part & 3), + 1 of lane half part >> 2 */
        uint4 *dst = lds.rows + buffer * kRows + (4 * (part & 3) + (vec >> 5)) * 64 + 32 * (part >> 2) + (vec & 31);
        uint32_t e = 0;
        float up = 1.f;
        if constexpr (Op::half) {
            float m = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[k][i]));
            e = half_exponent(over_parts_max(m)); /* of the vector's eight parts */
            up = __uint_as_float(e << 23);
            if (part == 0) sUnscale[buffer][vec] = half_unscale<NTERMS>(e);
        }
        float n2 = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = f[k][i] * up;
                n2 = __builtin_fmaf(x, x, n2);
            }
        n2 = over_parts_sum(n2);
        /* |x|^2 as the products give it: with the 2^15 of two terms of S, or the sqrt(d) of entries +-1 */
        if (part == 0) sNorm2[buffer][vec] = n2 * (NTERMS == 2 ? 0x1p30f : (NTERMS == 1 ? 128.f : 1.f));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            BOperand t[NXT];
            if constexpr (Op::half) split_half(f[k], e, t);
            else split_bf16(f[k], t);
#pragma unroll
            for (int x = 0; x < NXT; ++x) dst[(8 * x + k) * 2 * 64] = t[x].q;
        }
    };

    Item it{(int)(first_item / per_tile), (int)(first_item % per_tile), 0, 0, 0, 0, 0, 0};
    look_up(it);
    if (!it.some) return;
    load_row(it);
    if (needs_turn(it)) {
        load_turn(it);
        __syncthreads();
    }
    BOperand sa[8][NTERMS]; /* requested behind the first rows */
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
        for (int k = 0; k < NTERMS; ++k) sa[ks][k].q = S_terms[((k * 4 + rt) * 8 + ks) * 64 + lane];
    leave_row(0, kind_of(it));
    Thresholds th = load_thresholds(*a.consts, NTERMS == 1 ? PQ_INV_SQRT_D : 1.0f);
    const float base_scale = th.radius_scale;
    UpperTables ut = {};
    if (DEEP) ut = load_upper_tables(*a.consts);
    const DoubtLevels levels = doubt_levels(*a.exact);
    if (GENERAL) {
        sLut[tid] = a.consts->lut1[tid];
        th.lut1 = sLut;
        if (tid < 17) sPseudo[tid] = a.exact->pseudo1_f[tid];
    }
    for (int i = tid; i < 2 * kChunkItems; i += kThreads) (&sDoubt[0][0])[i] = 0;
    if (tid == 0) sCount = 0;
    const int tau = 32 * v + j;
    Item next = following(it);
    if (next.some) load_row(next);
    __syncthreads();
    if (needs_turn(next)) {
        load_turn(next);
        __syncthreads();
    }
    int n_done = 0;
    /* buffers are used in turn: what a wavefront writes for the tile after the next is behind the next tile's barrier */
    for (int turn = 0, storer = 0;; turn ^= 1, storer = (storer + 1) & 7, ++n_done) {
        const int lo = it.lo, hi = it.hi, kind = kind_of(it);
        const bool full = lo == 0 && hi == 64, valid = tau >= lo && tau < hi;
        const int64_t plane_tile = (int64_t)head_of(it) * a.table.pool_pages + it.page;
        uint8_t *gcodes = a.codes[kind] + plane_tile * PQL_CODE_BYTES;
        uint16_t *gradii = a.radii[kind] + plane_tile * kRadiiHalves;
        uint32_t *img = sImg[turn];
        if (tid == 0) sItem[n_done] = ChunkItem{it.page, it.row0, it.token0, 2 * head_of(it) + kind};
        if (!full) { /* the tile's present contents */
            const uint32_t *gc = reinterpret_cast<const uint32_t *>(gcodes);
            const uint32_t *gr = reinterpret_cast<const uint32_t *>(gradii);
            for (int c = tid; c < PQL_CODE_BYTES / 4; c += kThreads) img[c] = gc[c];
            for (int c = tid; c < kRadiiHalves / 2; c += kThreads) img[PQL_CODE_BYTES / 4 + c] = gr[c];
            __syncthreads();
        }
        if (Op::half) th.radius_scale = base_scale * sUnscale[turn][tau];
        auto mark = [&](bool doubt) { /* once per vector, whichever of its codes it is */
            if (!doubt || !valid) return;
            const uint32_t bit = 1u << j;
            if (atomicOr(&sDoubt[n_done][v], bit) & bit) return;
            const int at = atomicAdd(&sCount, 1);
            if (at < kListed) sList[at] = (uint32_t)n_done << 6 | (uint32_t)tau;
        };
        if (32 * v < hi && 32 * v + 32 > lo) {
            f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                BOperand xb[NXT];
#pragma unroll
                for (int x = 0; x < NXT; ++x) xb[x].q = lds.rows[turn * kRows + ((x * 8 + ks) * 2 + v) * 64 + lane];
#pragma unroll
                for (int term = NTERMS - 1; term >= 0; --term)
#pragma unroll
                    for (int x = 0; x < NXT; ++x)
                        if (x + term <= Op::top) acc = multiply<PQ_F32, NTERMS>(sa[ks][term], xb[x], acc);
            }
            bool doubt;
            const BlockCodes bc = quant_block_checked<GENERAL>(acc, th, doubt_of(sNorm2[turn][tau], levels), levels, sPseudo, doubt);
            mark(doubt);
            if (kind == PQ_KEY) {
                if (full) leave_block<PQ_KEY, DEEP>(img, tau, 4 * H + rt, bc);
                else if (valid) emit_block<PQ_KEY, DEEP>(img, tau, 4 * H + rt, bc);
            } else {
                if (full) leave_block<PQ_VALUE, DEEP>(img, tau, 4 * H + rt, bc);
                else if (valid) emit_block<PQ_VALUE, DEEP>(img, tau, 4 * H + rt, bc);
            }
            if (DEEP) sQ4[turn][v][rt][lane] = bc.q4;
        }
        const bool more = next.some;
        Item after = next;
        if (more) {
            leave_row(turn ^ 1, kind_of(next));
            after = following(next);
            if (after.some) load_row(after);
        }
        __syncthreads();
        if (more && needs_turn(after)) { /* the rows of the tile before have been turned */
            load_turn(after);
            __syncthreads();
        }
        if (DEEP && rt == 3 && 32 * v < hi && 32 * v + 32 > lo) {
            float q4[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q4[k] = sQ4[turn][v][k][lane];
            const UpperHalf mine = polar_upper_half(q4, H, ut);
            UpperHalf far;
            far.codes = from_other_half(mine.codes, H);
            far.q6 = __uint_as_float(from_other_half(__float_as_uint(mine.q6), H));
            const uint32_t word = H == 0 ? polar_upper_join(mine, far, th.radius_scale, ut) : polar_upper_join(far, mine, th.radius_scale, ut);
            const float err = kDoubt * __builtin_amdgcn_sqrtf(sNorm2[turn][tau]);
            const PqExact &E = *a.exact;
            mark(upper_in_doubt(q4[0], q4[1], ut.tan2[0], E.doubt[3], (1 << ut.b5) - 1, err) ||
                 upper_in_doubt(q4[2], q4[3], ut.tan2[0], E.doubt[3], (1 << ut.b5) - 1, err) ||
                 upper_in_doubt(q4[0] + q4[1], q4[2] + q4[3], ut.tan2[1], E.doubt[4], (1 << ut.b6) - 1, err) ||
                 upper_in_doubt(H == 0 ? mine.q6 : far.q6, H == 0 ? far.q6 : mine.q6, ut.tan2[2], E.doubt[5], (1 << ut.b7) - 1, err));
            if (H == 0 && valid) {
                if (full) reinterpret_cast<uint32_t *>(gradii)[tau] = word;
                else img[PQL_CODE_BYTES / 4 + tau] = word;
            }
        }
        if (full) {
            if (wave == storer) {
                if (kind == PQ_KEY) store_tile<PQ_KEY, DEEP>(img, gcodes, gradii, lane);
                else store_tile<PQ_VALUE, DEEP>(img, gcodes, gradii, lane);
            }
        } else {
            if (DEEP) __syncthreads();
            const uint4 *src = reinterpret_cast<const uint4 *>(img);
            for (int c = tid; c < kImgDwords / 4; c += kThreads) {
                if (c < PQL_CODE_BYTES / 16) reinterpret_cast<uint4 *>(gcodes)[c] = src[c];
                else reinterpret_cast<uint4 *>(gradii)[c - PQL_CODE_BYTES / 16] = src[c];
            }
        }
        if (!more) break;
        it = next;
        next = after;
    }
    ++n_done;

    /* ---- the vectors in doubt in 64 bits, one per wavefront and turn.  More than the list holds: lists are made from the marks, 256 vectors at a time. ---- */
    __syncthreads(); /* the workgroup's stores of whole tiles come before its updates of single fields */
    const int in_doubt = sCount;
    for (int skip = 0; skip < in_doubt; skip += kListed) {
        if (in_doubt > kListed) {
            __syncthreads();
            if (wave == 0) {
                int rank = 0; /* of the first marked vector of the 64 tiles */
                for (int base = 0; base < n_done; base += 64) {
                    const int i = base + lane;
                    uint64_t m = i < n_done ? (uint64_t)sDoubt[i][1] << 32 | sDoubt[i][0] : 0ull;
                    int incl = __popcll(m);
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) {
                        const int up = __shfl_up(incl, d);
                        if (lane >= d) incl += up;
                    }
                    for (int at = rank + incl - __popcll(m) - skip; m; m &= m - 1, ++at)
                        if (at >= 0 && at < kListed) sList[at] = (uint32_t)i << 6 | (uint32_t)__builtin_ctzll(m);
                    rank += __shfl(incl, 63);
                }
            }
            __syncthreads();
        }
        const int n = min(in_doubt - skip, kListed);
        for (int k = 0; k < n; k += 8) {
            ExactSlice s;
            s.load(a.exact->S, tid);
            ExactBounds bounds;
            bounds.load(*a.exact, *a.consts);
            const uint32_t entry = __builtin_amdgcn_readfirstlane(sList[min(k + wave, n - 1)]);
            const ChunkItem ci = sItem[entry >> 6];
            const int slot = (int)(entry & 63u), kind = ci.head_kind & 1, head = ci.head_kind >> 1;
            const int64_t row = (int64_t)ci.row0 + slot, off = row * a.ld_token + (int64_t)head * a.ld_head;
            const int64_t position = a.positions ? (int64_t)a.positions[row] : (int64_t)ci.token0 + slot;
            const double x0 = element_exact<XT>(a, kind, off, position, lane), x1 = element_exact<XT>(a, kind, off, position, lane + 64);
            lds.exact.x[wave][lane] = x0;
            lds.exact.x[wave][lane + 64] = x1;
            __syncthreads();
            if (n - k == 1) multiply_exact<1>(s, lds.exact, tid);
            else if (n - k <= 4) multiply_exact<4>(s, lds.exact, tid);
            else multiply_exact<8>(s, lds.exact, tid);
            __syncthreads();
            if (k + wave < n) {
                const double ya = rotated_exact(lds.exact, wave, 2 * lane), yb = rotated_exact(lds.exact, wave, 2 * lane + 1);
                const int64_t tile = (int64_t)head * a.table.pool_pages + ci.page;
                if (kind == PQ_KEY) write_exact<PQ_KEY>(a, bounds, ya, yb, tile, slot, lane);
                else write_exact<PQ_VALUE>(a, bounds, ya, yb, tile, slot, lane);
            }
            __syncthreads();
        }
    }
}

template <int XT>
void launch_chunks(const pq_ctx *ctx, const PqDeviceState *ds, const AppendPagedArgs &a, hipStream_t s)
{
    const int64_t n_items = 2 * (int64_t)a.n_heads * paged_tile_numbers(a.rows.n_rows, a.rows.n_seq);
    int64_t blocks = n_items < 256 ? n_items : 256; /* one workgroup per CU */
    if (n_items > blocks * kChunkItems) blocks = (n_items + kChunkItems - 1) / kChunkItems;
    auto launch = [&](auto kernel) {
        const uint16_t *terms = ctx->unit_entries || ctx->mixing ? ds->S_f16x2 : ds->S_bf16x3;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(512), 0, s, a, reinterpret_cast<const uint4 *>(terms), n_items);
    };
    auto with = [&](auto general, auto deep) {
        constexpr bool G = decltype(general)::value, D = decltype(deep)::value;
        if (ctx->unit_entries) launch(pq_append_chunk_kernel<XT, 1, G, D>);
        else if (ctx->mixing) launch(pq_append_chunk_kernel<XT, 2, G, D>);
        else launch(pq_append_chunk_kernel<XT, 3, G, D>);
    };
    auto with_books = [&](auto deep) {
        if (ctx->general_codebooks) with(std::true_type{}, deep);
        else with(std::false_type{}, deep);
    };
    if (ctx->depth == 7) with_books(std::true_type{});
    else with_books(std::false_type{});
}

} // namespace

extern "C" pq_status pq_append_paged(const pq_ctx *ctx, const void *xk, const void *xv, pq_dtype xt, int64_t n_rows, int n_heads,
                                     int64_t ld_token, int64_t ld_head, const pq_rotary *rotary, const int32_t *positions,
                                     uint8_t *k_codes, uint16_t *k_radii, uint8_t *v_codes, uint16_t *v_radii, int64_t pool_tokens,
                                     const int32_t *pages, int64_t ld_pages, const int32_t *row_start, const int32_t *ctx_len, int n_seq,
                                     void *hip_stream)
{
    if (!ctx) return PQ_EINVAL;
    if (n_rows == 0 || n_seq == 0) return PQ_OK;
    if (!xk || !xv || !k_codes || !k_radii || !v_codes || !v_radii || !pages || !row_start || !ctx_len) return PQ_EINVAL;
    if (xt != PQ_F32 && xt != PQ_BF16) return PQ_EINVAL;
    if (n_rows < 0 || n_seq < 0 || n_heads <= 0 || pool_tokens <= 0 || (pool_tokens & 63) || ld_pages <= 0) return PQ_EINVAL;
    if (ld_token < 0 || ld_head < 0) return PQ_EINVAL;
    if (n_rows > 0x7FFFFFFF / 2 / n_heads || n_seq > (1 << 29) || pool_tokens / 64 > 0x7FFFFFFF) return PQ_EUNSUPPORTED;
    const pq_status rs = pq_check_rotary(rotary);
    if (rs != PQ_OK) return rs;
    const int64_t elems16 = xt == PQ_BF16 ? 8 : 4;
    if (!pq_aligned16(xk) || !pq_aligned16(xv) || !pq_aligned16(k_codes) || !pq_aligned16(k_radii) || !pq_aligned16(v_codes) ||
        !pq_aligned16(v_radii) || (ld_token % elems16) || (ld_head % elems16))
        return PQ_EALIGN;
    const PqDeviceState *ds = nullptr;
    const pq_status st = pq_device_state(ctx, &ds);
    if (st != PQ_OK) return st;
    AppendPagedArgs a{{xk, xv}, {k_codes, v_codes}, {k_radii, v_radii}, ld_token, ld_head, n_heads,
                      PagedTable{pages, ld_pages, pool_tokens / 64}, PagedRows{row_start, ctx_len, n_seq, n_rows},
                      pq_rotary_args(rotary), positions, ds->exact, ds->consts};
    const int64_t n_vec = n_rows * n_heads;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    /* Whole tiles or vectors one by one: a vector takes 2.6 ns beyond the first two thousand, a tile that is written in part 17 ns
       and one number of a tile for every sequence whether it has tokens in it or not, the first of them 6 us more (heads x sequences x tokens
       each, us, vectors / tiles: 8 x 1 x 128 14.6 / 15.2, 256 21 / 14; 8 x 64 x 8 32 / 43, 16 50 / 45; 8 x 256 x 8 88 / 140, 16 167 / 156;
       2 x 64 x 8 14.5 / 16.6, 16 21 / 18; 2 x 1 x 256 11.3 / 13.4). */
    if (n_rows >= 12 * (int64_t)n_seq + 1024 / n_heads) {
        if (xt == PQ_BF16) launch_chunks<PQ_BF16>(ctx, ds, a, s);
        else launch_chunks<PQ_F32>(ctx, ds, a, s);
        PQ_HIP_TRY(hipGetLastError());
        return PQ_OK;
    }
    /* more than two workgroups per CU take four at a time: eight, and S stays in registers from the first to the last of them (8 x 64 x 8: 39 us
       with S fetched for every four, 32 so; 8 x 64 x 16 72 and 50; 8 x 256 x 1 25 and 19) */
    const int nv = n_vec > 4 * 256 ? 8 : append_vectors_per_block(2 * n_vec);
    const int n_blocks = (int)min((n_vec + nv - 1) / nv, (int64_t)256); /* two workgroups per CU, keys and values; 128 registers allow them */
    const dim3 grid(2u * (unsigned)n_blocks), block(512);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, n_vec, n_blocks); };
    auto with = [&](auto type) {
        constexpr int XT = decltype(type)::value;
        if (nv == 1) launch(pq_append_paged_kernel<XT, 1>);
        else if (nv == 4) launch(pq_append_paged_kernel<XT, 4>);
        else launch(pq_append_paged_kernel<XT, 8>);
    };
    if (xt == PQ_BF16) with(std::integral_constant<int, PQ_BF16>{});
    else with(std::integral_constant<int, PQ_F32>{});
    PQ_HIP_TRY(hipGetLastError());
    return PQ_OK;
}
