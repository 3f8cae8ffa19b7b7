/*
 * pq_paged.hip -- pq_append_paged: the keys and values of a ragged batch of new tokens to a paged cache, with the
 * position rotation of the keys on the way (Algorithm 1 lines 2 and 4 on k' = Rot(position) k and on v).
 *
 * Codes are settled in double precision: y = k' S with S, the rotation's products and the sums in 64 bits, and the
 * cell comparisons v > tan(t) u of procedure Quant as well (their squares above level 1).  A vector therefore gets
 * the codes of the definition whatever batch it comes in, and equal prefixes have equal pages.
 */
#include "pq_common.h"
#include "pq_polar.h"
#include "pq_paged.h"

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
__device__ __forceinline__ uint32_t level1_exact(double ya, double yb, const PqExact &E, bool general)
{
    const uint32_t sa = (uint32_t)(__double2hiint(ya)) >> 31, sb = (uint32_t)(__double2hiint(yb)) >> 31, f = sa ^ sb;
    const double a = fabs(ya), b = fabs(yb);
    if (!general) return (quant3_exact(a, b, E.tan1) ^ (f ? 7u : 0u)) | (sb << 3);
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

__device__ __forceinline__ double shfl_xor_double(double x, int d)
{
    const int lo = __shfl_xor(__double2loint(x), d), hi = __shfl_xor(__double2hiint(x), d);
    return __hiloint2double(hi, lo);
}

/* One rotated vector, coordinates 2 p and 2 p + 1 in lane p, to slot tau of a page: the recursion of procedure Polar with the codes'
 * comparisons, the nodes above level 1 in the lanes of their first leaf (the others compute the same along). */
template <int KIND>
__device__ __forceinline__ void write_exact(const AppendPagedArgs &a, double ya, double yb, int64_t tile, int tau, int lane)
{
    const PqExact &E = *a.exact;
    const PqDeviceConsts &K = *a.consts;
    const int i = lane & 7, b = lane >> 3;
    const uint32_t code1 = level1_exact(ya, yb, E, K.general != 0);
    const double q1 = ya * ya + yb * yb, q1s = shfl_xor_double(q1, 1);
    const uint32_t c2 = quant3_exact(q1, q1s, E.tan2[0]);
    const double q2 = q1 + q1s, q2s = shfl_xor_double(q2, 2);
    const uint32_t c3 = quant3_exact(q2, q2s, E.tan2[1]);
    const double q3 = q2 + q2s, q3s = shfl_xor_double(q3, 4);
    PqBlockFields f;
    f.c4 = quant3_exact(q3, q3s, E.tan2[2]);
    const double q4 = q3 + q3s;
    f.radius = radius_exact(q4);
    /* level-1 codes at their nibbles; [c2(2h) | c3(h) | c2(2h+1)] of half-block h at bits [8 h, 8 h + 6) */
    uint32_t l1 = code1 << (4 * i);
    uint32_t gw = (i & 1) ? 0u : ((i & 2) ? c2 : ((c2 << 4) | (c3 << 2))) << (2 * (i & 4));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        l1 |= __shfl_xor(l1, d);
        gw |= __shfl_xor(gw, d);
    }
    f.l1 = l1;
    f.g6[0] = gw & 63u;
    f.g6[1] = (gw >> 8) & 63u;
    if (i == 0) {
        pql_put_block<true>(reinterpret_cast<uint32_t *>(a.codes[KIND] + tile * PQL_CODE_BYTES), KIND, tau, b, f);
        if (K.depth != 7) a.radii[KIND][tile * PQL_RADII + pql_pos(KIND, tau, b).radius_half] = f.radius;
    }
    if (K.depth == 7) { /* levels 5, 6, 7 over the block radii, and the vector's word of the radius plane */
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

/* NV vectors (row, head) of kind KIND by one workgroup of 512 threads, vec0 .. vec0 + NV - 1 as far as they are below n_vec: S is fetched
 * once for the NV products (128 KB, what bounds the launch), a wavefront per vector then runs the recursion. */
template <int XT, int KIND, int NV>
__device__ __forceinline__ void append_vectors_exact(const AppendPagedArgs &a, int64_t vec0, int64_t n_vec, double (&sx)[4][PQ_D],
                                                     double (&spart)[4][4][PQ_D])
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kq = tid >> 7, j = tid & 127;
    double m[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) m[k] = a.exact->S[(32 * kq + k) * PQ_D + j];
    /* wavefronts 2 r and 2 r + 1 fetch vector r; a vector beyond the range repeats the last one and is not written */
    const int r = min(wave >> 1, NV - 1);
    const int64_t vec = min(vec0 + r, n_vec - 1), row = vec / a.n_heads;
    const int head = (int)(vec - row * a.n_heads);
    const PagedPlace at = paged_place(a, row, lane);
    if ((wave >> 1) < NV) {
        const int c = tid & 127;
        const int64_t off = row * a.ld_token + (int64_t)head * a.ld_head;
        auto element = [&](int k) -> double {
            if (XT == PQ_BF16) return (double)__uint_as_float((uint32_t) static_cast<const uint16_t *>(a.x[KIND])[off + k] << 16);
            return (double)static_cast<const float *>(a.x[KIND])[off + k];
        };
        double x = element(c);
        if (KIND == PQ_KEY && c < a.rot.dim) {
            const RotaryPair p = rotary_pair(a.rot, c);
            const float *cs = rotary_row(a.rot, at.position);
            const double s = (double)cs[(a.rot.dim >> 1) + p.at] * element(p.partner);
            x = x * (double)cs[p.at] + (p.minus ? -s : s);
        }
        sx[r][c] = x;
    }
    __syncthreads();
    {
        double acc[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) acc[v] = 0.0;
#pragma unroll
        for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int v = 0; v < NV; ++v) acc[v] = fma(sx[v][32 * kq + k], m[k], acc[v]);
#pragma unroll
        for (int v = 0; v < NV; ++v) spart[v][kq][j] = acc[v];
    }
    __syncthreads();
    if ((wave & 1) == 0 && (wave >> 1) < NV && vec0 + r < n_vec && at.page >= 0) {
        auto sum = [&](int c) { return ((spart[r][0][c] + spart[r][1][c]) + spart[r][2][c]) + spart[r][3][c]; };
        write_exact<KIND>(a, sum(2 * lane), sum(2 * lane + 1), head * a.table.pool_pages + at.page, at.tau, lane);
    }
}

/* workgroups [0, n_blocks): keys, the rest: values */
template <int XT, int NV>
__global__ __launch_bounds__(512) void pq_append_paged_kernel(AppendPagedArgs a, int64_t n_vec, int n_blocks)
{
    __shared__ double sx[4][PQ_D];
    __shared__ double spart[4][4][PQ_D];
    const int blk = (int)blockIdx.x;
    if (blk < n_blocks) append_vectors_exact<XT, PQ_KEY, NV>(a, (int64_t)NV * blk, n_vec, sx, spart);
    else append_vectors_exact<XT, PQ_VALUE, NV>(a, (int64_t)NV * (blk - n_blocks), n_vec, sx, spart);
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
    if (n_rows > 0x7FFFFFFF / 2 / n_heads || pool_tokens / 64 > 0x7FFFFFFF) return PQ_EUNSUPPORTED;
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
    const int nv = append_vectors_per_block(2 * n_vec);
    const int n_blocks = (int)((n_vec + nv - 1) / nv);
    const dim3 grid(2u * (unsigned)n_blocks), block(512);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, n_vec, n_blocks); };
    if (xt == PQ_BF16) nv == 1 ? launch(pq_append_paged_kernel<PQ_BF16, 1>) : launch(pq_append_paged_kernel<PQ_BF16, 4>);
    else nv == 1 ? launch(pq_append_paged_kernel<PQ_F32, 1>) : launch(pq_append_paged_kernel<PQ_F32, 4>);
    PQ_HIP_TRY(hipGetLastError());
    return PQ_OK;
}
