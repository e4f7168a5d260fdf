// Weight-streaming GEMM with weights in 4 bits.
//
//   C[m,n] = act(sum_k A[m,k] s[n,k/g] (q[n,k] - z[n,k/g]) + bias[n]) + residual[m,n]
// computed group by group as s (sum_k A q - z sum_k A), whose products are exact: q is 0 .. 15, a bf16 value; fp32
// rows of A are three bf16 planes hi + mid + lo (8 + 8 + 8 significant bits).  Sums are held in fp32.
//
// Codes lie as the products read them: [tiles of 16 rows][chunks of 128 k][4 pieces][16 rows][16 bytes], so that a
// wavefront's 16-byte load is 1 KB of consecutive memory and gives lane (row r, piece p) the codes of k = 32 t + 8 p + i,
// t = 0 .. 3 (dword t), i = 0 .. 7: the operand of four MFMAs 16x16x32.  Byte j of a dword holds i = j in its low and
// i = j + 4 in its high half.  As e4m3 the bytes 0 .. 15 are 0 .. 15 times 2^-9, so a conversion instruction turns two
// codes into two bf16 values.  Scales and zero points are bf16 [tiles][groups][16 rows].
//
// Bound by the bytes of the codes; sum_k A of a group is one more product, with a column operand of ones, so it comes
// out in the accumulators' layout.  A workgroup owns 16 NB columns; its wavefronts cut K into ranges of whole chunks
// and their partial tiles are added in wavefront order.
#include "gemm_common.hpp"

namespace lithos {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct GemmQ4Args {
    GemmArgs g;                 // A, C, bias, residual, sizes, flags of the epilogue
    const uint4* codes;
    const uint16_t* scales;
    const uint16_t* zeros;      // nullptr: 8
    int chunks, groups, gsteps; // chunks of 128 k; scale groups of a row; products (32 k) of a group: 1, 2 or 4
};

constexpr int Q4_WAVES = 8;

__device__ __forceinline__ bf16x8 q4_frag(uint32_t w)
{
    const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
    return __builtin_bit_cast(bf16x8, r);
}

__device__ __forceinline__ bf16x8 upper_halves(const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) w[p] = __builtin_amdgcn_perm(__float_as_uint(v[2 * p + 1]), __float_as_uint(v[2 * p]), 0x07060302u);
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

template <int MB, int NB, bool A32>
__global__ __launch_bounds__(Q4_WAVES * 64) void gemm_q4_kernel(GemmQ4Args a, AtomArgs atom)
{
    constexpr int NP = A32 ? 3 : 1;
    __shared__ __attribute__((aligned(16))) float red[Q4_WAVES][MB][NB][64][4];

    const GemmArgs& g = a.g;
    const Block3 blk = atom_delinearize(atom_logical_block(atom), atom);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kg = lane >> 4;
    const int m0 = blk.y * 16 * MB;
    const bool glu = NB == 2 && (g.flags & LITHOS_F_GLU);
    int tile[NB];                                    // GLU: gate rows' tile, up rows' tile
#pragma unroll
    for (int j = 0; j < NB; ++j) tile[j] = glu ? (int)blk.x + j * (g.N / 16) : min((int)blk.x * NB + j, (g.N + 15) / 16 - 1);
    const int c0 = (int)((int64_t)wave * a.chunks / Q4_WAVES), c1 = (int)((int64_t)(wave + 1) * a.chunks / Q4_WAVES);

    f32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));

    for (int c = c0; c < c1; ++c) {
        uint4 w[NB];
        float sc[NB], zc[NB];                        // of the group of this lane's piece of 32 k
        const int grp = min((4 * c + kg) / a.gsteps, a.groups - 1);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            w[j] = a.codes[((int64_t)tile[j] * a.chunks + c) * 64 + lane];
            const int64_t at = ((int64_t)tile[j] * a.groups + grp) * 16 + r16;
            sc[j] = bf16_to_f32(a.scales[at]);
            zc[j] = a.zeros ? bf16_to_f32(a.zeros[at]) : 8.0f;
        }
        f32x4 part[MB][NB], sum[MB];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t % a.gsteps == 0) {
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < NB; ++j) part[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
            const int k = 128 * c + 32 * t + 8 * kg, kc = min(k, g.K - 8);
            bf16x8 wf[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) wf[j] = q4_frag(t == 0 ? w[j].x : t == 1 ? w[j].y : t == 2 ? w[j].z : w[j].w);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const int64_t at = (int64_t)min(m0 + 16 * i + r16, g.M - 1) * g.lda + kc;
                bf16x8 xf[NP];
                if constexpr (A32) {
                    const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(g.A) + at);
                    const uint4 u = p[0], v = p[1];
                    const uint32_t raw[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
                    float x[8], r1[8], r2[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = k < g.K ? __uint_as_float(raw[e]) : 0.0f;
                        r1[e] = x[e] - __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);       // exact
                        r2[e] = r1[e] - __uint_as_float(__float_as_uint(r1[e]) & 0xffff0000u);     // exact, at most 8 bits
                    }
                    xf[0] = upper_halves(x); xf[1] = upper_halves(r1); xf[2] = upper_halves(r2);
                } else {
                    const uint4 u = *reinterpret_cast<const uint4*>(g.A + at);
                    xf[0] = __builtin_bit_cast(bf16x8, k < g.K ? u : make_uint4(0, 0, 0, 0));
                }
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[p], ones, sum[i], 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < NB; ++j) part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[p], wf[j], part[i][j], 0, 0, 0);
                }
            }
            if ((t + 1) % a.gsteps == 0) {
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    // the group of product t is that of piece t
                    const float s = __shfl(sc[j], 16 * t + r16), z = __shfl(zc[j], 16 * t + r16);
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, fmaf(-z, sum[i][e], part[i][j][e]), acc[i][j][e]);
                }
            }
        }
    }

#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4*>(&red[wave][i][j][lane][0]) = acc[i][j];
    __syncthreads();
    // element e of lane (r, p) is row 4 p + e, column r of its 16 x 16 block
    constexpr int OUT = MB * (NB * 256);
    for (int o = tid; o < (glu ? OUT / 2 : OUT); o += Q4_WAVES * 64) {
        const int i = glu ? o / 256 : o / (NB * 256), j = glu ? 0 : o / 256 % NB, l = o % 256 / 4, e = o % 4;
        float v = red[0][i][j][l][e];
#pragma unroll
        for (int w = 1; w < Q4_WAVES; ++w) v += red[w][i][j][l][e];
        if (glu) {
            float up = red[0][i][NB - 1][l][e];
#pragma unroll
            for (int w = 1; w < Q4_WAVES; ++w) up += red[w][i][NB - 1][l][e];
            v = v / (1.0f + expf(-v)) * up;
        }
        epilogue_store(g, m0 + 16 * i + 4 * (l >> 4) + e, ((int)blk.x * (glu ? 1 : NB) + j) * 16 + (l & 15), v);
    }
}

// ---- host side ----------------------------------------------------------------------

typedef void (*gemm_q4_fn)(GemmQ4Args, AtomArgs);

static gemm_q4_fn q4_kernel(const lithos_op_t& op)
{
    const bool a32 = op.flags & LITHOS_F_IN_F32;
    if (op.dim[0] > 16) return a32 ? gemm_q4_kernel<2, 2, true> : gemm_q4_kernel<2, 2, false>;
    return a32 ? gemm_q4_kernel<1, 2, true> : gemm_q4_kernel<1, 2, false>;
}

int gemm_q4_plan(const lithos_op_t& op, OpPlan* plan)
{
    const int64_t M = op.dim[0], N = op.dim[1], K = op.dim[2], group = op.dim[3];
    const int64_t lda = op.ld[0], ldc = op.ld[2], ldr = op.ld[3];
    const bool a32 = op.flags & LITHOS_F_IN_F32, glu = op.flags & LITHOS_F_GLU;
    if (M <= 0 || N <= 0 || K <= 0 || M > (1 << 24) || N > (1 << 28) || K > (1 << 28))
        return fail(LITHOS_EINVAL, "gemm_q4: M,N,K must be positive (got %lld,%lld,%lld)", (long long)M, (long long)N, (long long)K);
    if (K % 8) return fail(LITHOS_EINVAL, "gemm_q4: K must be a multiple of 8 (got %lld)", (long long)K);
    if (group != 32 && group != 64 && group != 128) return fail(LITHOS_EINVAL, "gemm_q4: groups of %lld k are not built (32, 64, 128)", (long long)group);
    if (op.flags & ~(LITHOS_F_BIAS | LITHOS_F_GELU | LITHOS_F_RESIDUAL | LITHOS_F_OUT_F32 | LITHOS_F_IN_F32 | LITHOS_F_GLU))
        return fail(LITHOS_EINVAL, "gemm_q4: takes BIAS, GELU, RESIDUAL, GLU, IN_F32 and OUT_F32 only");
    if (!op.in[0] || !op.in[1] || !op.in[4] || !op.out[0]) return fail(LITHOS_EINVAL, "gemm_q4: null operand");
    if (!aligned16(op.in[0]) || !aligned16(op.in[1]) || !aligned16(op.in[4]) || !aligned16(op.in[5]))
        return fail(LITHOS_EINVAL, "gemm_q4: A, codes, scales and zeros must be 16-byte aligned");
    if (!aligned_to(op.in[2], 4) || !aligned_to(op.in[3], 4) || !aligned_to(op.out[0], op.flags & LITHOS_F_OUT_F32 ? 4 : 2))
        return fail(LITHOS_EINVAL, "gemm_q4: misaligned bias, residual or output");
    if (lda < K || ldc < N || lda % (a32 ? 4 : 8)) return fail(LITHOS_EINVAL, "gemm_q4: leading dimension smaller than the row, or rows of A not 16-byte aligned");
    if ((op.flags & LITHOS_F_BIAS) && !op.in[2]) return fail(LITHOS_EINVAL, "gemm_q4: BIAS set but in[2] is null");
    if ((op.flags & LITHOS_F_RESIDUAL) && (!op.in[3] || ldr < N)) return fail(LITHOS_EINVAL, "gemm_q4: RESIDUAL needs in[3] and ldr >= N");
    if (glu && (op.flags & (LITHOS_F_BIAS | LITHOS_F_GELU | LITHOS_F_RESIDUAL))) return fail(LITHOS_EINVAL, "gemm_q4: GLU takes no BIAS, GELU or RESIDUAL");
    if (glu && N % 16) return fail(LITHOS_EINVAL, "gemm_q4: GLU needs N %% 16 == 0 (gate and up rows in tiles of their own)");
    const int64_t gx = glu ? N / 16 : (N + 31) / 32, gy = M > 16 ? (M + 31) / 32 : 1;
    if (gx * gy > 0x7fffffff) return fail(LITHOS_EINVAL, "gemm_q4: too many workgroups");
    plan->grid = {(uint32_t)gx, (uint32_t)gy, 1};
    plan->total = (uint32_t)(gx * gy);
    plan->threads = Q4_WAVES * 64;
    plan->variant = 0;
    plan->wg_per_cu = cached_occupancy((const void*)q4_kernel(op), (int)plan->threads, 2);
    return LITHOS_OK;
}

int gemm_q4_launch(const lithos_op_t& op, const OpPlan& plan, const AtomArgs& atom, hipStream_t s)
{
    GemmQ4Args a{};
    GemmArgs& g = a.g;
    g.A = (const uint16_t*)op.in[0];
    g.C = op.out[0];
    g.bias = (const float*)op.in[2];
    g.resid = (const float*)op.in[3];
    g.M = (int)op.dim[0]; g.N = (int)op.dim[1]; g.K = (int)op.dim[2];
    g.lda = op.ld[0]; g.ldc = op.ld[2]; g.ldr = op.ld[3];
    g.flags = op.flags;
    a.codes = (const uint4*)op.in[1];
    a.scales = (const uint16_t*)op.in[4];
    a.zeros = (const uint16_t*)op.in[5];
    a.chunks = (g.K + 127) / 128;
    a.groups = (int)((g.K + op.dim[3] - 1) / op.dim[3]);
    a.gsteps = (int)op.dim[3] / 32;
    LITHOS_HIP(launch_kernel(q4_kernel(op), dim3(LITHOS_ATOM_LAUNCH_BLOCKS(atom)), dim3(plan.threads), s, a, atom));
    return LITHOS_OK;
}

} // namespace lithos
