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
// Bound by the bytes of the codes where the vector ALUs keep up, which turn 1 KB of codes (a tile's chunk) into operands
// with some 30 instructions per lane and, for fp32 rows, split 128 k of A with up to 220: a workgroup owns NB 16-column
// blocks that share the latter.  Its eight wavefronts cut K into ranges of whole chunks; their partial tiles are added
// in wavefront order.  sum_k A of a group is one more product, with a column operand of ones, so it comes out in the
// accumulators' layout.  Scales and zero points come four groups of all tiles at a time, one 16-byte load per lane, and
// pass through the wavefront's own piece of LDS (a load of their own for each tile and chunk took as long as the codes).
// Measured: 1 x 4096 x 4096 in 4.9 us, 8 rows against 2 x 14336 x 4096 with gated SiLU in 20.7 us (66 MB, 3.2 TB/s), 27 x 5003 x
// 2088 bf16 in 9.0 us.  What a CU fetches bounds the latter two: the rows, 128 KB for each of 224 workgroups and 113 KB for each
// of 157, and loads behind a wavefront's range, which are issued (clamped to its last chunk) and not used: the caches are asked for
// 136 MB where 95 are needed, and for 51 where 24 are.  More rows than one operand holds cost the weights again: 32 fp32 rows x 6144 x
// 4096 13.3 us (bf16 rows 9.1), 512 bf16 rows x 4096 x 4096 44 us.
#pragma once
#include "gemm_common.hpp"

namespace lithos {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct GemmQ4Args {
    GemmArgs g;                 // A, C, bias, residual, sizes, flags of the epilogue
    const uint4* codes;
    const uint16_t* scales;
    const uint16_t* zeros;      // nullptr: 8
    int chunks, groups;         // chunks of 128 k, scale groups of a row
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

// fp32 values as three bf16 planes, exactly
template <int N>
__device__ __forceinline__ void residues(const float (&x)[N], float (&r1)[N], float (&r2)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        r1[e] = x[e] - __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
        r2[e] = r1[e] - __uint_as_float(__float_as_uint(r1[e]) & 0xffff0000u);      // at most 8 bits
    }
}

// workgroups per CU that registers and LDS are shared by
constexpr int q4_resident(int rows, int blocks, bool a32) { return blocks <= 2 && (rows <= 4 || (rows == 16 && !a32)) ? 2 : 1; }

// MR rows of A per workgroup (fp32: 2, 4, 8 or 16; bf16: 4, 16 or 32), NB 16-column blocks, GS products (32 k) to a group.
// A wavefront loads the live rows of a chunk as they lie, 256 or 512 bytes of a row together, splits fp32 ones once, and
// keeps the planes in its own piece of LDS, from which the row operands are read.  (Loads in the operands' layout touch 16
// rows each, whose stride is a power of two as a rule: 16 x 4096 x 4096 took 12 us with them.)  The row operand has room
// for 16 rows: it holds all three planes of up to 4 rows, two of 8 (the third then with zeros), one of 16; the planes' sums
// stay apart until the end.  Codes are D chunks ahead, A one (of 8 rows two: there it is most of what is in flight).
template <int MR, int NB, int GS, bool A32>
__global__ __launch_bounds__(Q4_WAVES * 64, 2 * q4_resident(MR, NB, A32))
void gemm_q4_kernel(GemmQ4Args a, AtomArgs atom)
{
    constexpr int MB = MR > 16 ? 2 : 1, D = NB == 1 ? 4 : 2, XD = NB == 1 && MR == 8 ? 2 : 1, NG = 4 / GS;
    constexpr int PLANES = A32 ? 3 : 1, PR = MR <= 4 ? 4 : MR == 8 ? 8 : 16;    // a plane's rows in an operand
    constexpr int PN = A32 ? 16 / PR : 1, NP = A32 ? (PLANES + PN - 1) / PN : 1; // planes in an operand, operands of 16 rows
    constexpr int EPL = A32 ? 4 : 8, NX = MR * 128 / (64 * EPL);                // elements per 16-byte load; loads per lane and chunk
    constexpr int ROW = 128 + 8, XROWS = PLANES * MR + 1;                       // padded rows of the planes, and one of zeros
    constexpr int XBYTES = Q4_WAVES * XROWS * ROW * 2, RBYTES = Q4_WAVES * MB * NB * 1024;
    static_assert(NX >= 1, "a chunk of A fills whole loads");
    __shared__ __attribute__((aligned(16))) unsigned char smem[XBYTES > RBYTES ? XBYTES : RBYTES];
    __shared__ __attribute__((aligned(16))) uint16_t factors[Q4_WAVES][2][NB * 4 * 16];   // scales, zeros: [tile][group][row]

    const GemmArgs& g = a.g;
    const Block3 blk = atom_delinearize(atom_logical_block(atom), atom);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kg = lane >> 4, m0 = blk.x * MR;       // row blocks that share weights are neighbours
    const bool glu = NB >= 2 && (g.flags & LITHOS_F_GLU);
    constexpr int H = NB >= 2 ? NB / 2 : 1;                                     // GLU: H tiles of gate rows, then the H tiles of their up rows
    const int ntiles = (g.N + 15) / 16;
    auto tile_of = [&](int j) { return glu ? min((int)blk.y * H + j % H, ntiles - 1) + j / H * ntiles : min((int)blk.y * NB + j, ntiles - 1); };
    const int c0 = (int)((int64_t)wave * a.chunks / Q4_WAVES), c1 = (int)((int64_t)(wave + 1) * a.chunks / Q4_WAVES);

    const uint4* codes[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) codes[j] = a.codes + (int64_t)tile_of(j) * a.chunks * 64 + lane;
    auto load_codes = [&](uint4 (&w)[NB], int c) {
#pragma unroll
        for (int j = 0; j < NB; ++j) w[j] = codes[j][(int64_t)min(c, c1 - 1) * 64];
    };

    // four groups from `first` on: lane (tile l / 8, group l / 2 % 4, half l % 2)
    const int64_t fbase = (int64_t)tile_of(min(lane / 8, NB - 1)) * a.groups;
    uint4 sreg, zreg = make_uint4(0x41004100u, 0x41004100u, 0x41004100u, 0x41004100u);     // 8
    auto load_factors = [&](int first) {
        const int64_t at = (fbase + min(first + lane / 2 % 4, a.groups - 1)) * 2 + lane % 2;
        sreg = reinterpret_cast<const uint4*>(a.scales)[at];
        if (a.zeros) zreg = reinterpret_cast<const uint4*>(a.zeros)[at];
    };
    uint16_t (*const fac)[NB * 4 * 16] = factors[wave];
    auto stage_factors = [&]() {
        if (lane < NB * 8) {
            reinterpret_cast<uint4*>(fac[0])[lane] = sreg;
            reinterpret_cast<uint4*>(fac[1])[lane] = zreg;
        }
    };

    uint4 raws[XD][NX];
    auto load_rows = [&](uint4 (&raw)[NX], int c) {
        c = min(c, c1 - 1);
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int f = (i * 64 + lane) * EPL;
            const int64_t at = (int64_t)min(m0 + f / 128, g.M - 1) * g.lda + min(128 * c + f % 128, g.K - EPL);
            if constexpr (A32) raw[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(g.A) + at);
            else raw[i] = *reinterpret_cast<const uint4*>(g.A + at);
        }
    };
    uint16_t* const xs = reinterpret_cast<uint16_t*>(smem) + wave * XROWS * ROW;
    if (lane < ROW / 4) *reinterpret_cast<uint2*>(xs + PLANES * MR * ROW + lane * 4) = make_uint2(0, 0);
    const uint16_t* xrow[MB][NP];                                               // this lane's row of each operand
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int o = 0; o < NP; ++o) {
            const int plane = o * PN + r16 / PR, m = 16 * i + r16 % PR;
            xrow[i][o] = xs + (plane < PLANES && m < MR ? plane * MR + m : PLANES * MR) * ROW + 8 * kg;
        }
    auto stage_rows = [&](const uint4 (&raw)[NX], int c) {
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int f = (i * 64 + lane) * EPL;
            const bool live = 128 * c + f % 128 < g.K;
            uint16_t* const dst = xs + (f / 128) * ROW + f % 128;
            if constexpr (A32) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                float x[4], r1[4], r2[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = live ? __uint_as_float(w[e]) : 0.0f;
                residues(x, r1, r2);
                auto put = [&](uint16_t* at, const float (&v)[4]) {
                    *reinterpret_cast<uint2*>(at) = make_uint2(__builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302u),
                                                               __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]), 0x07060302u));
                };
                put(dst, x); put(dst + MR * ROW, r1); put(dst + 2 * MR * ROW, r2);
            } else {
                *reinterpret_cast<uint4*>(dst) = live ? raw[i] : make_uint4(0, 0, 0, 0);
            }
        }
    };

    f32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));

    if (c0 < c1) {
        uint4 w[D][NB];
#pragma unroll
        for (int d = 0; d < XD; ++d) load_rows(raws[d], c0 + d);
        load_factors(c0 * NG);
#pragma unroll
        for (int d = 0; d < D; ++d) load_codes(w[d], c0 + d);
        for (int cb = c0; cb < c1; cb += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const int c = cb + d;
                if (c >= c1) break;
                wave_lds_sync();                                                // what the last chunk read from LDS it has read
                if (((c - c0) & (GS - 1)) == 0) {
                    stage_factors();
                    load_factors((c + GS) * NG);
                }
                stage_rows(raws[d % XD], c);
                load_rows(raws[d % XD], c + XD);
                wave_lds_sync();
                const int fg = ((c - c0) & (GS - 1)) * NG;                      // the chunk's first group among the four
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    bf16x8 xf[4][NP];
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int o = 0; o < NP; ++o) xf[t][o] = *reinterpret_cast<const bf16x8*>(xrow[i][o] + 32 * t);
                    f32x4 sum[NG];
#pragma unroll
                    for (int q = 0; q < NG; ++q) {
                        sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int t = q * GS; t < (q + 1) * GS; ++t)
#pragma unroll
                            for (int p = NP - 1; p >= 0; --p) sum[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t][p], ones, sum[q], 0, 0, 0);
                    }
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const uint32_t wj[4] = {w[d][j].x, w[d][j].y, w[d][j].z, w[d][j].w};
#pragma unroll
                        for (int q = 0; q < NG; ++q) {
                            f32x4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int t = q * GS; t < (q + 1) * GS; ++t) {
                                const bf16x8 wf = q4_frag(wj[t]);
#pragma unroll
                                for (int p = NP - 1; p >= 0; --p) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t][p], wf, part, 0, 0, 0);
                            }
                            const int at = (j * 4 + fg + q) * 16 + r16;
                            const float s = bf16_to_f32(fac[0][at]), z = bf16_to_f32(fac[1][at]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, fmaf(-z, sum[q][e], part[e]), acc[i][j][e]);
                        }
                        // two tiles overlap; left alone, the scheduler starts all of them and runs out of registers
                        if (j % 2) __builtin_amdgcn_sched_barrier(0);
                    }
                }
                load_codes(w[d], c + D);
            }
        }
    }

    __syncthreads();                                 // the planes give way to the partial tiles
    float (*red)[MB][NB][64][4] = reinterpret_cast<float (*)[MB][NB][64][4]>(smem);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4*>(&red[wave][i][j][lane][0]) = acc[i][j];
    __syncthreads();
    // element e of lane (r, p) is row 4 p + e, column r of its 16 x 16 block; neighbouring threads take neighbouring columns
    const int nc = glu ? H : NB;                     // 16-column blocks of C
    auto total = [&](int r, int j, int col) {
        float v = 0.0f;
#pragma unroll
        for (int p = PN - 1; p >= 0; --p)            // the small planes first
#pragma unroll
            for (int u = 0; u < Q4_WAVES; ++u) {
                const int row = r % 16 + p * PR;
                if (p >= PLANES) continue;
                v += red[u][r / 16][j][row / 4 * 16 + col][row % 4];
            }
        return v;
    };
    for (int o = tid; o < MR * nc * 16; o += Q4_WAVES * 64) {
        const int col = o % (nc * 16), r = o / (nc * 16);
        if (m0 + r >= g.M) break;
        float v = total(r, col / 16, col % 16);
        if (glu) v = v / (1.0f + expf(-v)) * total(r, col / 16 + H, col % 16);
        epilogue_store(g, m0 + r, (int)blk.y * nc * 16 + col, v);
    }
}

typedef void (*gemm_q4_fn)(GemmQ4Args, AtomArgs);

// rows: 2, 4, 8, 16 (fp32), 4, 16, 32 (bf16); blocks: 1, 2, 4, 8 (2, 4 and 32 rows: at most 4)
template <int GS, int NB>
static gemm_q4_fn q4_pick(int rows, bool a32)
{
    constexpr int FEW = NB == 8 ? 4 : NB;
    if (!a32) return rows == 4 ? gemm_q4_kernel<4, FEW, GS, false> : rows == 16 ? gemm_q4_kernel<16, NB, GS, false> : gemm_q4_kernel<32, FEW, GS, false>;
    return rows == 2 ? gemm_q4_kernel<2, FEW, GS, true> : rows == 4 ? gemm_q4_kernel<4, FEW, GS, true>
         : rows == 8 ? gemm_q4_kernel<8, NB, GS, true> : gemm_q4_kernel<16, NB, GS, true>;
}

template <int GS>
static gemm_q4_fn q4_table(int rows, int blocks, bool a32)
{
    return blocks == 8 ? q4_pick<GS, 8>(rows, a32) : blocks == 4 ? q4_pick<GS, 4>(rows, a32) : blocks == 2 ? q4_pick<GS, 2>(rows, a32) : q4_pick<GS, 1>(rows, a32);
}

gemm_q4_fn gemm_q4_g32_fn(int rows, int blocks, bool a32);
gemm_q4_fn gemm_q4_g64_fn(int rows, int blocks, bool a32);
gemm_q4_fn gemm_q4_g128_fn(int rows, int blocks, bool a32);

} // namespace lithos
