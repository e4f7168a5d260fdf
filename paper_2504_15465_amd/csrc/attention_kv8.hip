// A key/value cache of 8 bits with one fp32 scale per block of positions and head, and the decode attention
// that reads it.
//
//  * kv8_append_kernel - quantises new keys and values into the cache (ROPE_KV's place in a chain).
//  * attn_dec8_kernel  - one query token per sequence, grouped-query, against that cache (ATTN_DEC's place).
//
// Cache: codes [batch, cap, n_kv, d] bytes (int8, or e4m3 with F_E4M3), keys and values apart; scales fp32
// [2, batch, ceil(cap / block), n_kv], keys' then values'.  A code c stands for scale * c.
#include "common.hpp"
#include <math.h>
#include <algorithm>

namespace lithos {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---- append -----------------------------------------------------------------------
// One wavefront per (sequence, block of positions that the new tokens touch, head, keys or values).
//   s_new = max |x| / Q         (Q = 127 for int8, 448 for e4m3; the quotient rounded to fp32)
// A block that starts with the new tokens takes s_new.  One that holds earlier positions keeps its scale s_old if
// that is at least s_new; otherwise its earlier codes c become round(fl(fl(c s_old) / s_new)).  New codes are
// round(fl(x / s)), 0 where s is 0 or no number.  Every step is an IEEE fp32 operation, so the result is defined to the bit.
// Bound by the bytes of the new rows (read twice, the second time from the cache) and codes.  A lane owns eight
// neighbouring elements of a row: 16-byte loads (two of them for fp32), 8-byte stores.
struct Kv8AppendArgs {
    const void* x[2];           // new keys, new values: row (b * T + t), head h at column h * d
    uint8_t* codes[2];
    float* scales;              // [2][batch][nblk][n_kv]
    const int32_t* positions;   // first position per sequence, or nullptr
    int64_t pos, ld;
    int batch, T, n_kv, cap, block, nblk, touched;
};

__device__ __forceinline__ uint32_t quantise4(const float (&x)[8], int at, float s, bool e4m3)
{
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = s > 0.0f && s < INFINITY ? x[at + e] / s : 0.0f;      // 0 times infinity reads as NaN
    if (e4m3) {
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fminf(fmaxf(y[e], -448.0f), 448.0f);       // beyond 464 the conversion gives NaN
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (uint32_t)((int)fminf(fmaxf(rintf(y[e]), -127.0f), 127.0f) & 0xff) << (8 * e);
    return w;
}

// byte e of w as the number that the code stands for
template <bool E4M3, int E>
__device__ __forceinline__ float code_value(uint32_t w)
{
    if constexpr (E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)w, E);
    else return (float)(int8_t)(w >> (8 * E));
}

template <bool E4M3>
__device__ __forceinline__ void code_values8(const uint2& w, float (&f)[8])
{
    f[0] = code_value<E4M3, 0>(w.x); f[1] = code_value<E4M3, 1>(w.x); f[2] = code_value<E4M3, 2>(w.x); f[3] = code_value<E4M3, 3>(w.x);
    f[4] = code_value<E4M3, 0>(w.y); f[5] = code_value<E4M3, 1>(w.y); f[6] = code_value<E4M3, 2>(w.y); f[7] = code_value<E4M3, 3>(w.y);
}

template <int D, bool X32, bool E4M3>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8AppendArgs a, AtomArgs atom)
{
    constexpr int LPR = D / 8, RPS = 64 / LPR;          // lanes per row, rows per step
    const uint32_t L = atom_logical_block(atom);
    const int64_t unit = (int64_t)L * 4 + (threadIdx.x >> 6);
    const int64_t units = 2ll * a.batch * a.touched * a.n_kv;
    if (unit >= units) return;
    const int lane = threadIdx.x & 63, c = (lane % LPR) * 8, r0 = lane / LPR;
    const int kv = unit & 1;
    const int h = (int)((unit >> 1) % a.n_kv), tb = (int)((unit >> 1) / a.n_kv % a.touched), b = (int)((unit >> 1) / a.n_kv / a.touched);
    const int64_t p0 = a.positions ? (int64_t)a.positions[b] : a.pos;
    if (p0 < 0) return;                                  // a sequence that takes no part
    const int64_t blk = p0 / a.block + tb;
    const int64_t first = blk * a.block;
    const int64_t lo = max(p0, first), hi = min(min(p0 + a.T, first + a.block), (int64_t)a.cap);
    if (lo >= hi) return;

    const int64_t esz = X32 ? 4 : 2;
    const char* src = reinterpret_cast<const char*>(a.x[kv]) + (((int64_t)b * a.T - p0) * a.ld + (int64_t)h * D + c) * esz;   // + position * ld
    auto load = [&](int64_t p, float (&x)[8]) {
        const uint4* at = reinterpret_cast<const uint4*>(src + p * a.ld * esz);
        const uint4 u = at[0];
        if constexpr (X32) {
            const uint4 v = at[1];
            const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
        } else {
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
        }
    };

    // largest magnitude as a bit pattern: a NaN counts as larger than everything and makes the scale NaN
    uint32_t top = 0;
    for (int64_t p = lo + r0; p < hi; p += RPS) {
        float x[8];
        load(p, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const float fresh = __uint_as_float(top) / (E4M3 ? 448.0f : 127.0f);

    float* const sp = a.scales + (((int64_t)kv * a.batch + b) * a.nblk + blk) * a.n_kv + h;
    uint8_t* const dst = a.codes[kv] + ((int64_t)b * a.cap * a.n_kv + h) * D + c;
    const int64_t row = (int64_t)a.n_kv * D;
    float s = fresh;
    if (lo > first) {
        const float old = *sp;
        const bool grown = !(fresh <= old) && old == old;       // a NaN scale stays
        s = grown ? fresh : old;
        if (grown)
            for (int64_t p = first + r0; p < lo; p += RPS) {
                uint2* at = reinterpret_cast<uint2*>(dst + p * row);
                float x[8];
                code_values8<E4M3>(*at, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= old;
                *at = make_uint2(quantise4(x, 0, s, E4M3), quantise4(x, 4, s, E4M3));
            }
    }
    if (lane == 0) *sp = s;
    for (int64_t p = lo + r0; p < hi; p += RPS) {
        float x[8];
        load(p, x);
        *reinterpret_cast<uint2*>(dst + p * row) = make_uint2(quantise4(x, 0, s, E4M3), quantise4(x, 4, s, E4M3));
    }
}

// ---- decode attention ---------------------------------------------------------------
//   o_h = sum_t p_ht vs_t vc_t / sum_t p_ht,   p_ht = exp(scale ks_t (q_h . kc_t) - max_t ...)
// with kc, vc the codes and ks, vs the scales of the position's block.  The cache is read once: bound by its bytes.
//
// A workgroup owns a range of keys of one (sequence, key/value head), its four wavefronts units of 32 keys each; the
// up to 16 query heads of the group are the column operand of MFMA 16x16x32 (columns beyond the group compute on zeros
// and are not stored).  The contraction index of a product may be numbered in any order that both operands share:
//  * scores S[key][head]: a lane (r = lane % 16, g = lane / 16) loads 16-byte pieces g, g + 4, .. of key row r, and
//    step t multiplies the 8 bytes at 64 (t / 2) + 16 g + 8 (t % 2): the codes go from memory to the operand registers;
//  * the result leaves a lane with the scores of head r and keys 4 g + e of both 16-key halves of the unit, which is the
//    column operand of the value product if its slot (g, i) is key 16 (i / 4) + 4 g + i % 4; the row operand is
//    V^T[d][key], and with d = (D / 16) r + j for product j a lane's piece of a value row is D / 16 bytes.
// So neither keys, values nor probabilities pass through LDS.  Codes become bf16 exactly.  fp32 queries are three bf16
// planes hi + mid + lo (exact); p vs is split into as many planes as the output has use for: three (exact) for fp32,
// two (2^-16) for bf16.  Scale factors are applied to sums and probabilities in fp32.
struct Dec8Args {
    const void* q;
    const uint8_t* k;
    const uint8_t* v;
    const float* scales;
    const int32_t* lens;        // keys per sequence, or nullptr: `keys` everywhere
    void* o;
    float* ws;
    int64_t ldq;
    float scale;
    int batch, n_q, n_kv, keys, cap, block, nblk, splits;
};

// two codes (bytes 2H, 2H + 1 of w) as bf16
template <bool E4M3, int H>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w)
{
    if constexpr (E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, H != 0));
    else return pack_bf16((float)(int8_t)(w >> (16 * H)), (float)(int8_t)(w >> (16 * H + 8)));
}

template <bool E4M3>
__device__ __forceinline__ bf16x8 codes_frag(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(bf16x8, make_uint4(codes_bf16<E4M3, 0>(a), codes_bf16<E4M3, 1>(a), codes_bf16<E4M3, 0>(b), codes_bf16<E4M3, 1>(b)));
}

// eight fp32 values as P bf16 planes by truncation, largest first
template <int P>
__device__ __forceinline__ void split_planes(const float (&x)[8], bf16x8 (&out)[P])
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(__float_as_uint(r[2 * e + 1]), __float_as_uint(r[2 * e]), 0x07060302u);
        out[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        if (p + 1 < P)
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] -= __uint_as_float(__float_as_uint(r[e]) & 0xffff0000u);      // exact
    }
}

template <int D>
struct Dec8Unit {
    uint4 k[2][D / 64];         // key rows r and 16 + r
    uint32_t v[8][D / 64];      // slot i's value row, D / 16 bytes
    float ks[2], vs[2];
};

template <int D, bool E4M3, bool Q32, bool O32>
__global__ __launch_bounds__(256, 2) void attn_dec8_kernel(Dec8Args a, AtomArgs atom)
{
    constexpr int NS = D / 32, QP = Q32 ? 3 : 1, PP = O32 ? 3 : 2, NV = D / 16, NW = D / 64;
    __shared__ __attribute__((aligned(16))) float part_o[4][16][D];
    __shared__ float part_m[4][16], part_l[4][16];

    const uint32_t L = atom_logical_block(atom);
    const int S = a.splits;
    const int g = L % a.n_kv, sp = (L / a.n_kv) % S, b = L / a.n_kv / S;
    const int G = a.n_q / a.n_kv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kg = lane >> 4;

    const int T = a.lens ? max(0, min(__builtin_amdgcn_readfirstlane(a.lens[b]), a.keys)) : a.keys;
    const int U = (T + 31) / 32;
    const int u0 = (int)((int64_t)sp * U / S), u1 = (int)((int64_t)(sp + 1) * U / S);

    // queries of the group, in the scores' contraction order
    bf16x8 qf[NS][QP];
#pragma unroll
    for (int t = 0; t < NS; ++t) {
        const int64_t at = (int64_t)b * a.ldq + (int64_t)(g * G + min(r16, G - 1)) * D + 64 * (t / 2) + 16 * kg + 8 * (t % 2);
        if constexpr (Q32) {
            const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(a.q) + at);
            const uint4 u = p[0], w = p[1];
            float x[8] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w),
                          __uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r16 < G ? x[e] : 0.0f;
            split_planes<QP>(x, qf[t]);
        } else {
            const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + at);
            qf[t][0] = __builtin_bit_cast(bf16x8, r16 < G ? u : make_uint4(0, 0, 0, 0));
        }
    }

    const uint32_t row = (uint32_t)a.n_kv * D;                       // bytes between positions
    const uint8_t* const kbase = a.k + ((int64_t)b * a.cap * a.n_kv + g) * D;
    const uint8_t* const vbase = a.v + ((int64_t)b * a.cap * a.n_kv + g) * D;
    const float* const ksc = a.scales + (int64_t)b * a.nblk * a.n_kv + g;
    const float* const vsc = ksc + (int64_t)a.batch * a.nblk * a.n_kv;

    typedef Dec8Unit<D> Unit;
    auto load = [&](Unit& x, int u) {
        u = min(u, U - 1);                                           // a unit beyond the range is loaded, not used
        const int last = T - 1 - 32 * u;                             // dead keys read the last live row
        const uint8_t* const kp = kbase + (int64_t)(32 * u) * row;
        const uint8_t* const vp = vbase + (int64_t)(32 * u) * row;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint32_t at = (uint32_t)min(16 * hf + r16, last) * row + 16 * kg;
#pragma unroll
            for (int c = 0; c < NW; ++c) x.k[hf][c] = *reinterpret_cast<const uint4*>(kp + at + 64 * c);
            const int64_t bl = (int64_t)(min(32 * u + 16 * hf, T - 1) / a.block) * a.n_kv;
            x.ks[hf] = ksc[bl];
            x.vs[hf] = vsc[bl];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t at = (uint32_t)min(16 * (i / 4) + 4 * kg + i % 4, last) * row + NV * r16;
            if constexpr (NW == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(vp + at);
                x.v[i][0] = w.x; x.v[i][1] = w.y;
            } else {
                x.v[i][0] = *reinterpret_cast<const uint32_t*>(vp + at);
            }
        }
    };

    float m = -INFINITY, l = 0.0f;             // of head r16: m the same in its four lanes, l over this lane's keys
    f32x4 acc[NV];                             // O^T: element e of product j is d = NV (4 kg + e) + j of head r16
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto compute = [&](const Unit& x, int u) {
        float s8[8];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const uint4 w = x.k[hf][t / 2];
                const bf16x8 kf = t % 2 ? codes_frag<E4M3>(w.z, w.w) : codes_frag<E4M3>(w.x, w.y);
#pragma unroll
                for (int p = QP - 1; p >= 0; --p) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][p], sc, 0, 0, 0);
            }
            const float f = a.scale * x.ks[hf];
#pragma unroll
            for (int e = 0; e < 4; ++e) s8[4 * hf + e] = 32 * u + 16 * hf + 4 * kg + e < T ? sc[e] * f : -INFINITY;
        }
        float bm = s8[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) bm = fmaxf(bm, s8[i]);
        bm = fmaxf(bm, __shfl_xor(bm, 16));
        bm = fmaxf(bm, __shfl_xor(bm, 32));
        const float nm = fmaxf(m, bm);
        const float ref = nm == -INFINITY ? 0.0f : nm;
        if (__any(nm > m)) {
            const float corr = expf(m - ref);                        // 0 while m = -inf
            l *= corr;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] *= corr;
            m = nm;
        }
        float p8[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = expf(s8[i] - ref);                       // 0 for a dead key
            l += p;
            p8[i] = p * x.vs[i / 4];
        }
        bf16x8 pf[PP];
        split_planes<PP>(p8, pf);
#pragma unroll
        for (int c = 0; c < NW; ++c) {
            auto product = [&](auto bb) {
                constexpr int B = decltype(bb)::value, j0 = 0;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = pack_bf16(code_value<E4M3, B>(x.v[2 * i][c]), code_value<E4M3, B>(x.v[2 * i + 1][c]));
                const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                const int j = j0 + 4 * c + B;
#pragma unroll
                for (int p = PP - 1; p >= 0; --p) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[p], acc[j], 0, 0, 0);
            };
            product(std::integral_constant<int, 0>{});
            product(std::integral_constant<int, 1>{});
            product(std::integral_constant<int, 2>{});
            product(std::integral_constant<int, 3>{});
        }
    };

    if (u0 + wave < u1) {
        Unit x0, x1;
        load(x0, u0 + wave);
        for (int u = u0 + wave; u < u1; u += 8) {
            load(x1, u + 4);
            compute(x0, u);
            if (u + 4 < u1) {
                load(x0, u + 8);
                compute(x1, u + 4);
            }
        }
    }

    // the wavefronts' partial softmaxes, merged in wavefront order
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (r16 < G) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NV; j += 4)
                *reinterpret_cast<float4*>(&part_o[wave][r16][NV * (4 * kg + e) + j]) = make_float4(acc[j][e], acc[j + 1][e], acc[j + 2][e], acc[j + 3][e]);
        if (kg == 0) { part_m[wave][r16] = m; part_l[wave][r16] = l; }
    }
    __syncthreads();
    for (int i = tid; i < G * D; i += 256) {
        const int h = i / D, d = i % D;
        float gm = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) gm = fmaxf(gm, part_m[w][h]);
        const float ref = gm == -INFINITY ? 0.0f : gm;               // no key: every partial is empty
        float num = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = expf(part_m[w][h] - ref);
            num += part_o[w][h][d] * f;
            den += part_l[w][h] * f;
        }
        if (S == 1) {
            const float r = den == 0.0f ? 0.0f : num / den;          // a sequence without keys: zeros
            const int64_t idx = (int64_t)b * ((int64_t)a.n_q * D) + (int64_t)(g * G + h) * D + d;
            if constexpr (O32) reinterpret_cast<float*>(a.o)[idx] = r;
            else reinterpret_cast<uint16_t*>(a.o)[idx] = f32_to_bf16(r);
        } else {
            const int64_t prow = (((int64_t)b * a.n_kv + g) * S + sp) * G + h;      // ATTN_MERGE's workspace
            a.ws[prow * D + d] = num;
            if (d == 0) {
                float* ml = a.ws + (int64_t)a.batch * a.n_q * S * D + prow * 2;
                ml[0] = gm;
                ml[1] = den;
            }
        }
    }
}

// ---- host side ----------------------------------------------------------------------

typedef void (*dec8_fn)(Dec8Args, AtomArgs);
typedef void (*append_fn)(Kv8AppendArgs, AtomArgs);

template <int D>
static dec8_fn dec8_pick(bool e4m3, bool q32, bool o32)
{
    if (e4m3) return q32 ? (o32 ? attn_dec8_kernel<D, true, true, true> : attn_dec8_kernel<D, true, true, false>)
                         : (o32 ? attn_dec8_kernel<D, true, false, true> : attn_dec8_kernel<D, true, false, false>);
    return q32 ? (o32 ? attn_dec8_kernel<D, false, true, true> : attn_dec8_kernel<D, false, true, false>)
               : (o32 ? attn_dec8_kernel<D, false, false, true> : attn_dec8_kernel<D, false, false, false>);
}

static dec8_fn dec8_kernel(const lithos_op_t& op)
{
    const bool e = op.flags & LITHOS_F_E4M3, q = op.flags & LITHOS_F_IN_F32, o = op.flags & LITHOS_F_OUT_F32;
    return op.dim[3] == 64 ? dec8_pick<64>(e, q, o) : dec8_pick<128>(e, q, o);
}

static append_fn append_kernel(const lithos_op_t& op)
{
    const bool e = op.flags & LITHOS_F_E4M3, x = op.flags & LITHOS_F_IN_F32;
    if (op.dim[3] == 64) return x ? (e ? kv8_append_kernel<64, true, true> : kv8_append_kernel<64, true, false>)
                                  : (e ? kv8_append_kernel<64, false, true> : kv8_append_kernel<64, false, false>);
    return x ? (e ? kv8_append_kernel<128, true, true> : kv8_append_kernel<128, true, false>)
             : (e ? kv8_append_kernel<128, false, true> : kv8_append_kernel<128, false, false>);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// blocks of positions that the new tokens of a sequence can touch
static int64_t touched_blocks(const lithos_op_t& op)
{
    const int64_t T = op.dim[1], pos = op.dim[4], block = op.dim[6];
    return op.in[2] ? (T + block - 2) / block + 1 : (pos + T - 1) / block - pos / block + 1;
}

static int check_cache(const char* who, int64_t batch, int64_t n_kv, int64_t d, int64_t cap, int64_t block)
{
    if (batch <= 0 || n_kv <= 0 || batch > (1 << 24) || n_kv > (1 << 16)) return fail(LITHOS_EINVAL, "%s: batch and key/value heads must be positive (got %lld, %lld)", who, (long long)batch, (long long)n_kv);
    if (d != 64 && d != 128) return fail(LITHOS_EINVAL, "%s: head width %lld is not built (64, 128)", who, (long long)d);
    if (cap <= 0 || cap > (1ll << 30)) return fail(LITHOS_EINVAL, "%s: cache capacity %lld", who, (long long)cap);
    if (block < 16 || block > 1024 || block % 16) return fail(LITHOS_EINVAL, "%s: a block of %lld positions is not built (multiples of 16 up to 1024)", who, (long long)block);
    return LITHOS_OK;
}

int kv8_plan(const lithos_op_t& op, OpPlan* plan)
{
    plan->threads = 256;
    plan->variant = 0;
    plan->wg_per_cu = 4;
    if (op.kind == LITHOS_OP_KV8_APPEND) {
        // dim = batch, tokens, n_kv, d, pos, cap, block
        const int64_t batch = op.dim[0], T = op.dim[1], n_kv = op.dim[2], d = op.dim[3], pos = op.dim[4], cap = op.dim[5], block = op.dim[6];
        const int rc = check_cache("kv8_append", batch, n_kv, d, cap, block);
        if (rc != LITHOS_OK) return rc;
        if (T <= 0 || T > cap) return fail(LITHOS_EINVAL, "kv8_append: need 0 < tokens <= cap (got %lld)", (long long)T);
        if (!op.in[2] && (pos < 0 || pos > cap - T)) return fail(LITHOS_EINVAL, "kv8_append: positions %lld .. %lld lie outside the cache", (long long)pos, (long long)(pos + T - 1));
        if (!op.in[0] || !op.in[1] || !op.in[3] || !op.out[0] || !op.out[1]) return fail(LITHOS_EINVAL, "kv8_append: null operand");
        const bool x32 = op.flags & LITHOS_F_IN_F32;
        if (!aligned16(op.in[0]) || !aligned16(op.in[1]) || !aligned16(op.out[0]) || !aligned16(op.out[1]))
            return fail(LITHOS_EINVAL, "kv8_append: keys, values and caches must be 16-byte aligned");
        if (!aligned_to(op.in[2], 4) || !aligned_to(op.in[3], 4)) return fail(LITHOS_EINVAL, "kv8_append: misaligned positions or scales");
        if (op.ld[0] < n_kv * d || op.ld[0] % (x32 ? 4 : 8)) return fail(LITHOS_EINVAL, "kv8_append: row stride %lld is smaller than n_kv*d or breaks the 16-byte alignment of rows", (long long)op.ld[0]);
        const int64_t units = 2 * batch * touched_blocks(op) * n_kv;
        if ((units + 3) / 4 > 0x7fffffff) return fail(LITHOS_EINVAL, "kv8_append: too many workgroups");
        plan->grid = {(uint32_t)((units + 3) / 4), 1, 1};
        plan->total = plan->grid.x;
        plan->wg_per_cu = cached_occupancy((const void*)append_kernel(op), 256, 4);
        return LITHOS_OK;
    }
    // ATTN_DEC8: dim = batch, n_q, n_kv, d, keys, cap, splits, block
    const int64_t batch = op.dim[0], n_q = op.dim[1], n_kv = op.dim[2], d = op.dim[3], keys = op.dim[4], cap = op.dim[5], block = op.dim[7];
    const int64_t splits = op.dim[6] > 0 ? op.dim[6] : 1;
    const int rc = check_cache("attn_dec8", batch, n_kv, d, cap, block);
    if (rc != LITHOS_OK) return rc;
    if (n_q <= 0 || n_q % n_kv || n_q / n_kv > 16) return fail(LITHOS_EINVAL, "attn_dec8: need 1 to 16 query heads per key/value head (got %lld and %lld)", (long long)n_q, (long long)n_kv);
    if (keys <= 0 || keys > cap) return fail(LITHOS_EINVAL, "attn_dec8: need 0 < keys <= cap");
    if (op.ld[0] < n_q * d) return fail(LITHOS_EINVAL, "attn_dec8: q row stride smaller than n_q*d");
    if (!op.in[0] || !op.in[1] || !op.in[2] || !op.in[4] || !op.out[0]) return fail(LITHOS_EINVAL, "attn_dec8: null operand");
    if (!aligned16(op.in[0]) || !aligned16(op.in[1]) || !aligned16(op.in[2]) || op.ld[0] % 8)
        return fail(LITHOS_EINVAL, "attn_dec8: q and the caches must be 16-byte aligned, q's row stride a multiple of 8");
    if (!aligned_to(op.in[4], 4) || !aligned_to(op.in[5], 4) || !aligned_to(op.out[0], op.flags & LITHOS_F_OUT_F32 ? 4 : 2))
        return fail(LITHOS_EINVAL, "attn_dec8: misaligned scales, lengths or output");
    if (splits > LITHOS_ATTN_MAX_SPLITS) return fail(LITHOS_EINVAL, "attn_dec8: splits %lld above %d", (long long)splits, LITHOS_ATTN_MAX_SPLITS);
    if (splits > 1 && (!op.in[3] || !aligned16(op.in[3]))) return fail(LITHOS_EINVAL, "attn_dec8: a split launch needs a 16-byte aligned workspace in in[3]");
    if (batch * n_kv * splits > 0x7fffffff) return fail(LITHOS_EINVAL, "attn_dec8: too many workgroups");
    plan->grid = {(uint32_t)(n_kv * splits), (uint32_t)batch, 1};
    plan->total = (uint32_t)(batch * n_kv * splits);
    plan->wg_per_cu = cached_occupancy((const void*)dec8_kernel(op), 256, 2);
    return LITHOS_OK;
}

int kv8_launch(const lithos_op_t& op, const OpPlan& plan, const AtomArgs& atom, hipStream_t s)
{
    const dim3 grid(LITHOS_ATOM_LAUNCH_BLOCKS(atom)), block(plan.threads);
    if (op.kind == LITHOS_OP_KV8_APPEND) {
        Kv8AppendArgs a{};
        a.x[0] = op.in[0]; a.x[1] = op.in[1];
        a.codes[0] = (uint8_t*)op.out[0]; a.codes[1] = (uint8_t*)op.out[1];
        a.scales = (float*)const_cast<void*>(op.in[3]);
        a.positions = (const int32_t*)op.in[2];
        a.batch = (int)op.dim[0]; a.T = (int)op.dim[1]; a.n_kv = (int)op.dim[2];
        a.pos = op.dim[4]; a.cap = (int)op.dim[5]; a.block = (int)op.dim[6];
        a.ld = op.ld[0];
        a.nblk = (int)ceil_div(a.cap, a.block);
        a.touched = (int)touched_blocks(op);
        LITHOS_HIP(launch_kernel(append_kernel(op), grid, block, s, a, atom));
        return LITHOS_OK;
    }
    Dec8Args a{};
    a.q = op.in[0]; a.k = (const uint8_t*)op.in[1]; a.v = (const uint8_t*)op.in[2];
    a.ws = (float*)const_cast<void*>(op.in[3]);
    a.scales = (const float*)op.in[4]; a.lens = (const int32_t*)op.in[5];
    a.o = op.out[0];
    a.ldq = op.ld[0]; a.scale = op.fparam[0];
    a.batch = (int)op.dim[0]; a.n_q = (int)op.dim[1]; a.n_kv = (int)op.dim[2];
    a.keys = (int)op.dim[4]; a.cap = (int)op.dim[5]; a.splits = op.dim[6] > 0 ? (int)op.dim[6] : 1; a.block = (int)op.dim[7];
    a.nblk = (int)ceil_div(a.cap, a.block);
    LITHOS_HIP(launch_kernel(dec8_kernel(op), grid, block, s, a, atom));
    return LITHOS_OK;
}

// Key ranges per (sequence, key/value head): two workgroups per CU of the target, of at least four units of 32 keys each
// (one per wavefront), so that a short sequence is not cut only to be joined again.
int kv8_split_hint(const lithos_op_t& op, int n_cus)
{
    const int64_t quads = ceil_div(op.dim[4], 128), want = ceil_div(2ll * n_cus, op.dim[0] * op.dim[2]);
    return (int)std::max<int64_t>(1, std::min({quads, want, (int64_t)LITHOS_ATTN_MAX_SPLITS}));
}

} // namespace lithos
