// GEMM_Q4: validation, kernel choice, launch.
#include "gemm_q4.hpp"

namespace lithos {

// ---- host side ----------------------------------------------------------------------

// rows of A per workgroup
static int q4_rows(const lithos_op_t& op)
{
    const int64_t M = op.dim[0];
    if (!(op.flags & LITHOS_F_IN_F32)) return M > 16 ? 32 : M > 4 ? 16 : 4;
    return M > 8 ? 16 : M > 4 ? 8 : M > 2 ? 4 : 2;
}

// 16-column blocks per workgroup.  More blocks share the loads and the splitting of A, which weigh about as much as x blocks;
// fewer fill the chip.  Time goes with the workgroups of a CU times blocks + x.  A value of C does not depend on the choice.
// Eight blocks of up to four rows are 12 % slower than four (1 x 2 x 14336 x 4096: 1, 2, 4, 8 blocks 19.5, 19.7, 18.0, 20.3 us
// a pass); 8 rows 30, 30, 25.5, 22.8, 16 rows 42, 42, 31.7, 26.5; 1 x 4096 x 4096 5.5, 6.2, 8.1, 12.7, 1 x 6144 x 4096 7.2, 6.5,
// 8.3, 12.8; 24 x 5003 x 2088 bf16 10.6, 8.7, 12.1.  The rule misses the best for 1 x 5003 x 2088: two blocks 6.2 us, one 5.6.  With
// eight blocks of 16 fp32 rows, groups of 32 spill two registers: 16 x 2 x 14336 x 4096 in groups of 32, 64, 128 k 32, 26, 25 us.
static int q4_blocks(const lithos_op_t& op)
{
    const bool glu = op.flags & LITHOS_F_GLU, a32 = op.flags & LITHOS_F_IN_F32;
    const int rows = q4_rows(op), x = !a32 ? (rows + 15) / 16 : rows == 16 ? 5 : rows == 8 ? 3 : 2;
    const int64_t tiles = (glu ? 2 : 1) * ((op.dim[1] + 15) / 16), gy = (op.dim[0] + rows - 1) / rows;
    int best = 0;
    int64_t least = 0;
    for (int nb = glu ? 2 : 1; nb <= (rows <= 4 || rows == 32 ? 4 : 8); nb *= 2) {
        const int64_t t = ((tiles + nb - 1) / nb * gy + 255) / 256 * (nb + x);
        if (!best || t < least) { best = nb; least = t; }
    }
    return best;
}

static gemm_q4_fn q4_kernel(const lithos_op_t& op)
{
    const bool a32 = op.flags & LITHOS_F_IN_F32;
    const int rows = q4_rows(op), nb = q4_blocks(op);
    return op.dim[3] == 32 ? gemm_q4_g32_fn(rows, nb, a32) : op.dim[3] == 64 ? gemm_q4_g64_fn(rows, nb, a32) : gemm_q4_g128_fn(rows, nb, a32);
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
    const int64_t cols = 16 * q4_blocks(op) / (glu ? 2 : 1), gx = (N + cols - 1) / cols, gy = (M + q4_rows(op) - 1) / q4_rows(op);
    if (gx * gy > 0x7fffffff) return fail(LITHOS_EINVAL, "gemm_q4: too many workgroups");
    plan->grid = {(uint32_t)gy, (uint32_t)gx, 1};
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
    LITHOS_HIP(launch_kernel(q4_kernel(op), dim3(LITHOS_ATOM_LAUNCH_BLOCKS(atom)), dim3(plan.threads), s, a, atom));
    return LITHOS_OK;
}

} // namespace lithos
