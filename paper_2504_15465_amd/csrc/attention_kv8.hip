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
// One wavefront, or of more than 16 tokens one workgroup, per (sequence, block of positions that the new tokens touch, head,
// keys or values).
//   s_new = max |x| / Q         (Q = 127 for int8, 448 for e4m3; the quotient rounded to fp32)
// A block that starts with the new tokens takes s_new.  One that holds earlier positions keeps its scale s_old if
// that is at least s_new; otherwise its earlier codes c become round(fl(fl(c s_old) / s_new)).  New codes are
// round(fl(x / s)), 0 where s is 0 or no number.  Every step is an IEEE fp32 operation, so the result is defined to the bit.
// Bound by the bytes of the new rows and codes; 64 rows of fp32 or 128 of bf16 stay in registers between the maximum
// and the codes, longer blocks are read twice: 8192 tokens of 8 heads of 128 bf16 take 12.9 us, 3.9 TB/s.  A lane owns eight
// neighbouring elements of a row: 16-byte loads (two of them for fp32), 8-byte stores.
struct Kv8AppendArgs {
    const void* x[2];           // new keys, new values: row (b * T + t), head h at column h * d
    uint8_t* codes[2];
    float* scales;              // [2][batch][nblk][n_kv]
    const int32_t* positions;   // first position per sequence, or nullptr
    int64_t pos, ld;
    int batch, T, n_kv, cap, block, nblk, touched;
};

// four quotients as codes
template <bool E4M3>
__device__ __forceinline__ uint32_t encode4(const float (&y)[8], int at)
{
    if constexpr (E4M3) {
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = __builtin_amdgcn_fmed3f(y[at + e], -448.0f, 448.0f);       // beyond 464 the conversion gives NaN
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
    }
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (uint32_t)((int)__builtin_amdgcn_fmed3f(rintf(y[at + e]), -127.0f, 127.0f) & 0xff) << (8 * e);
    return w;
}

// codes of eight elements.  The quotient by a scale of ordinary size takes two corrections with its rounded reciprocal: the
// first leaves it within one unit of the last place, the second, whose remainder is exact, rounds it correctly (P. Markstein,
// 1990), in five instructions where the division takes eleven.  Elements so small that a remainder would not be exact have
// code 0 either way.  (The remainder is s y - x, not x - s y: for x = -0 the latter would add +0 and lose the sign, which e4m3 keeps.)
template <bool E4M3>
__device__ __forceinline__ uint2 quantise8(const float (&x)[8], float s, float rcp)
{
    float y[8];
    if (s >= 0x1p-60f && s <= 0x1p60f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = x[e] * rcp;
            y[e] = fmaf(fmaf(s, y[e], -x[e]), -rcp, y[e]);
            y[e] = fmaf(fmaf(s, y[e], -x[e]), -rcp, y[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = s > 0.0f && s < INFINITY ? x[e] / s : 0.0f;                  // 0 times infinity reads as NaN
    }
    return make_uint2(encode4<E4M3>(y, 0), encode4<E4M3>(y, 4));
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

template <int D, bool X32, bool E4M3, int WPU>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8AppendArgs a, AtomArgs atom)
{
    constexpr int LPR = D / 8, RPS = 64 / LPR * WPU, STEPS = WPU == 1 ? 1 : X32 ? 4 : 8;      // lanes per row, rows per step, steps in registers
    __shared__ uint32_t tops[4];
    const uint32_t L = atom_logical_block(atom);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t unit = WPU == 4 ? (int64_t)L : (int64_t)L * 4 + wave;
    const int64_t units = 2ll * a.batch * a.touched * a.n_kv;
    if (unit >= units) return;                           // of a unit per wavefront; there are no barriers then
    const int c = (lane % LPR) * 8, r0 = lane / LPR + (WPU == 4 ? wave * (64 / LPR) : 0);
    const int kv = unit & 1;
    const uint32_t pair = (uint32_t)(unit >> 1), block_of = pair / (uint32_t)a.n_kv;          // below 2^32; divisions of 64 bits are long
    const int h = (int)(pair % (uint32_t)a.n_kv), tb = (int)(block_of % (uint32_t)a.touched), b = (int)(block_of / (uint32_t)a.touched);
    const int64_t p0 = a.positions ? (int64_t)a.positions[b] : a.pos;
    if (p0 < 0) return;                                  // a sequence that takes no part
    const uint32_t blk = (uint32_t)p0 / (uint32_t)a.block + tb;                               // p0 < 2^31
    const int64_t first = (int64_t)blk * a.block;
    const int64_t lo = max(p0, first), hi = min(min(p0 + a.T, first + a.block), (int64_t)a.cap);
    if (lo >= hi) return;
    const int n = (int)(hi - lo), held = (int)(lo - first);      // new positions, earlier ones

    constexpr int64_t esz = X32 ? 4 : 2;
    const char* const src = reinterpret_cast<const char*>(a.x[kv]) + (((int64_t)b * a.T + (lo - p0)) * a.ld + (int64_t)h * D + c) * esz;
    struct Raw { uint4 u[X32 ? 2 : 1]; } raw[STEPS];
    auto load = [&](int base) {                          // rows beyond the last repeat it
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const uint4* at = reinterpret_cast<const uint4*>(src + (int64_t)min(base + i * RPS + r0, n - 1) * a.ld * esz);
#pragma unroll
            for (int e = 0; e < (X32 ? 2 : 1); ++e) raw[i].u[e] = at[e];
        }
    };
    auto unpack = [&](const Raw& r, float (&x)[8]) {
        if constexpr (X32) {
            const uint32_t w[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[X32].x, r.u[X32].y, r.u[X32].z, r.u[X32].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
        } else {
            const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
        }
    };

    float* const sp = a.scales + (((int64_t)kv * a.batch + b) * a.nblk + blk) * a.n_kv + h;
    const float old = held ? *sp : 0.0f;
    // largest magnitude as a bit pattern: a NaN counts as larger than everything and makes the scale NaN
    uint32_t top = 0;
    for (int base = (n - 1) / (STEPS * RPS) * (STEPS * RPS); base >= 0; base -= STEPS * RPS) {
        load(base);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float x[8];
            unpack(raw[i], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        }
    }
    top = lane_group<64>(top, [](uint32_t x, uint32_t y) { return max(x, y); });
    if constexpr (WPU == 4) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    const float fresh = __uint_as_float(top) / (E4M3 ? 448.0f : 127.0f);
    const bool grown = held && !(fresh <= old) && old == old;    // a NaN scale stays
    const float s = held && !grown ? old : fresh, rcp = 1.0f / s;

    const int64_t row = (int64_t)a.n_kv * D;
    uint8_t* const dst = a.codes[kv] + (((int64_t)b * a.cap + first) * a.n_kv + h) * D + c;
    if (grown)
        for (int p = r0; p < held; p += RPS) {
            uint2* at = reinterpret_cast<uint2*>(dst + p * row);
            float x[8];
            code_values8<E4M3>(*at, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= old;
            *at = quantise8<E4M3>(x, s, rcp);
        }
    if (lane == 0 && (WPU == 1 || wave == 0) && (!held || grown)) *sp = s;
    for (int base = 0; base < n; base += STEPS * RPS) {
        if (base) load(base);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int p = base + i * RPS + r0;
            float x[8];
            unpack(raw[i], x);
            if (p < n) *reinterpret_cast<uint2*>(dst + (held + p) * row) = quantise8<E4M3>(x, s, rcp);
        }
    }
}

// ---- decode attention ---------------------------------------------------------------
//   o_h = sum_t p_ht vs_t vc_t / sum_t p_ht,   p_ht = exp(scale ks_t (q_h . kc_t) - max_t ...)
// with kc, vc the codes and ks, vs the scales of the position's block.  The cache is read once: bound by its bytes, or for
// short sequences by the latencies of one pass.
//
// A workgroup owns a range of keys of one (sequence, key/value head), its wavefronts units of 32 keys each.  The
// contraction index of a product may be numbered in any order that both operands share:
//  * scores S[key][column] = keys x queries on MFMA 16x16x32: a lane (r = lane % 16, g = lane / 16) loads 16-byte pieces
//    g, g + 4, .. of key row r, and step t multiplies the 8 bytes at 64 (t / 2) + 16 g + 8 (t % 2): the codes go from
//    memory to the operand registers;
//  * the result leaves a lane with the scores of its column and keys 4 g + e of both 16-key halves of the unit, which is
//    the column operand of the value product if its slot (g, i) is key 16 (i / 4) + 4 g + i % 4; the row operand is
//    V^T[d][key], and with d = (D / 16) r + j for product j a lane's piece of a value row is D / 16 bytes.
// So neither keys, values nor probabilities pass through LDS.  Codes become bf16 exactly.  fp32 queries are three bf16
// planes hi + mid + lo (exact); p vs is split into as many planes as the output has use for: three (exact) for fp32, for bf16
// two, each rounded to nearest (2^-18 at worst, without a preferred side; cut off after 16 bits, outputs were low by 2^-17 on
// average: 0.6 % of those of 8 sequences of 32768 keys were not the exact result's rounding, now 0.26 %, in the same time).  The 16 columns hold CS heads (4, 8 or 16, the group rounded up) of 16 / CS planes, so that a
// group of up to four heads takes one product where 16 heads take one per plane; the planes' scores are added across the
// columns, and the accumulators at the end.  Scale factors are applied to sums and probabilities in fp32; exponents are
// powers of two.  Measured: 8 sequences of 32768 keys, 8 heads of 64, in 56 us (4.8 TB/s), 16 ragged ones of up to 2049 keys,
// 8 heads of 128, in 14 us (34 MB; an empty launch takes 3), one of 300 keys in 7.4 us.
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
    int batch, n_q, n_kv, keys, nblk, splits;
    int64_t seq;                // bytes of a sequence's keys
    uint32_t blk_magic;         // ceil(2^32 / (block / 16)), 0 for 16
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

// the upper halves of eight fp32 values: bf16, truncated
__device__ __forceinline__ bf16x8 upper_halves(const float (&r)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(__float_as_uint(r[2 * e + 1]), __float_as_uint(r[2 * e]), 0x07060302u);
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

// Plane `plane` of x as an operand: x less the planes before it, truncated.  `steps` planes come before the lowest one of
// the lanes, `most` before the highest.  Behind the third plane of 24 bits nothing is left.
template <int STEPS, int MOST>
__device__ __forceinline__ bf16x8 plane_operand(const float (&x)[8], int plane)
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int s = 0; s < MOST && s < 2; ++s) {
        const uint32_t mask = s < STEPS || plane > s ? 0xffff0000u : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] -= __uint_as_float(__float_as_uint(r[e]) & mask);             // exact
    }
    return upper_halves(r);
}

// x as bf16, or with `second` what the rounding left of it as bf16 (the difference is exact); both rounded to nearest
__device__ __forceinline__ bf16x8 rounded_operand(const float (&x)[8], bool second)
{
    const uint32_t lo = second ? 0xffff0000u : 0u;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t first = pack_bf16(x[2 * e], x[2 * e + 1]);
        w[e] = pack_bf16(x[2 * e] - __uint_as_float((first << 16) & lo), x[2 * e + 1] - __uint_as_float(first & lo));
    }
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

// the sum over the 16 / CS columns of a head, in every one of them
template <int CS>
__device__ __forceinline__ float slot_sum(float x)
{
    if constexpr (CS <= 8) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, true));      // row_ror:8
    if constexpr (CS <= 4) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x124, 0xf, 0xf, true));      // row_ror:4
    return x;
}

template <int D>
struct Dec8Unit {
    uint4 k[2][D / 64];         // key rows r and 16 + r
    uint32_t v[8][D / 64];      // slot i's value row, D / 16 bytes
    float ks[2], vs[2];
};

constexpr float DEC8_LOG2E = 1.44269504088896340736f, DEC8_LN2 = 0.69314718055994530942f;

// W wavefronts: eight share a few long ranges, which one CU would take long to fetch; four, where blocks are many, let two
// workgroups (heads of 64: four) overlap on a CU.
template <int D, bool E4M3, bool Q32, bool O32, int CS, int W>
__global__ __launch_bounds__(W * 64, 2) void attn_dec8_kernel(Dec8Args a, AtomArgs atom)
{
    constexpr int NS = D / 32, NV = D / 16, NW = D / 64, PPO = 16 / CS;
    constexpr int QP = Q32 ? 3 : 1, PP = O32 ? 3 : 2, NQ = (QP + PPO - 1) / PPO, NP = (PP + PPO - 1) / PPO;
    __shared__ __attribute__((aligned(16))) float part_o[W][CS][D];
    __shared__ float part_m[W][CS], part_l[W][CS];

    const uint32_t L = atom_logical_block(atom);
    const int S = a.splits;
    // sequences run fastest, turned by one each time: a die's contiguous share of the blocks then holds as much of a long
    // sequence as the others', and blocks that meet on a CU are of different ones
    uint32_t turn = L, b = 0, g = 0, sp = 0;                          // divisions only where there is something to divide
    if (a.batch > 1) { turn = L / a.batch; b = (L % a.batch + turn) % a.batch; }
    if (turn < (uint32_t)a.n_kv) g = turn;
    else { sp = turn / a.n_kv; g = turn % a.n_kv; }
    const int G = a.n_q / a.n_kv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kg = lane >> 4, head = r16 % CS, slot = r16 / CS;

    const int T = a.lens ? max(0, min(__builtin_amdgcn_readfirstlane(a.lens[b]), a.keys)) : a.keys;
    const int U = (T + 31) / 32;
    const int u0 = S == 1 ? 0 : (int)(sp * (uint32_t)U / (uint32_t)S), u1 = S == 1 ? U : (int)((sp + 1) * (uint32_t)U / (uint32_t)S);   // 64 * 2^25 at most

    const uint32_t row = (uint32_t)a.n_kv * D;                       // bytes between positions
    const uint8_t* const kbase = a.k + (int64_t)b * a.seq + g * D;
    const uint8_t* const vbase = a.v + (int64_t)b * a.seq + g * D;
    typedef const __attribute__((address_space(4))) float* uniform_ptr;           // read through the scalar cache
    const uniform_ptr ksc = (uniform_ptr)(a.scales + (int64_t)b * a.nblk * a.n_kv + g), vsc = ksc + (int64_t)a.batch * a.nblk * a.n_kv;

    typedef Dec8Unit<D> Unit;
    const uint32_t kat = (uint32_t)r16 * row + 16 * kg, vat = (uint32_t)(4 * kg) * row + NV * r16;
    auto load_at = [&](Unit& x, const uint8_t* kp, const uint8_t* vp, auto&& koff, auto&& voff) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int c = 0; c < NW; ++c) x.k[hf][c] = *reinterpret_cast<const uint4*>(koff(kp, hf) + 64 * c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (NW == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(voff(vp, i));
                x.v[i][0] = w.x; x.v[i][1] = w.y;
            } else {
                x.v[i][0] = *reinterpret_cast<const uint32_t*>(voff(vp, i));
            }
        }
    };
    auto load = [&](Unit& x, int u) {
        u = min(u, U - 1);                                           // a unit beyond the range is loaded, not used
        const int last = T - 1 - 32 * u;
        const uint8_t* const kp = kbase + (int64_t)(32 * u) * row;
        const uint8_t* const vp = vbase + (int64_t)(32 * u) * row;
        // The two cases are kept apart (the empty assembly): joined, every unit would compute the last one's addresses.
        if (last >= 31) {                                            // one lane offset, the rows in the scalar base
            load_at(x, kp, vp, [&](const uint8_t* q, int hf) { return q + (int64_t)(16 * hf) * row + kat; },
                    [&](const uint8_t* q, int i) { return q + (int64_t)(16 * (i / 4) + i % 4) * row + vat; });
            asm volatile("; whole unit");
        } else {                                                     // dead keys read the last live row
            load_at(x, kp, vp, [&](const uint8_t* q, int hf) { return q + (uint32_t)min(16 * hf + r16, last) * row + 16 * kg; },
                    [&](const uint8_t* q, int i) { return q + (uint32_t)min(16 * (i / 4) + 4 * kg + i % 4, last) * row + NV * r16; });
            asm volatile("; last unit");
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint32_t half = 2 * u + (16 * hf <= last ? hf : 0);
            const int64_t bl = (int64_t)(a.blk_magic ? __umulhi(half, a.blk_magic) : half) * a.n_kv;
            x.ks[hf] = ksc[bl];
            x.vs[hf] = vsc[bl];
        }
    };
    Unit x0, x1;
    const bool busy = u0 + wave < u1;
    if (busy) { load(x0, u0 + wave); load(x1, u0 + wave + W); }

    // The queries' planes, split once for all wavefronts: column c of operand o holds plane o * PPO + c / CS of head c % CS (a
    // single plane stands in every slot), in the scores' contraction order.
    __shared__ __attribute__((aligned(16))) uint16_t qs[NQ][16][D + 8];
    for (int i = tid; i < NQ * 16 * (D / 8); i += W * 64) {
        const int c8 = i % (D / 8), col = i / (D / 8) % 16, o = i / (D / 8) / 16;
        const int h = col % CS, plane = QP == 1 ? 0 : o * PPO + col / CS;
        const int64_t at = (int64_t)b * a.ldq + (int64_t)(g * G + min(h, G - 1)) * D + 8 * c8;
        const bool live = h < G && plane < QP;
        bf16x8 f;
        if constexpr (Q32) {
            const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(a.q) + at);
            const uint4 u = p[0], w = p[1];
            const float x[8] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w),
                                __uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
            f = plane_operand<0, 2>(x, plane);
        } else {
            f = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + at));
        }
        *reinterpret_cast<uint4*>(&qs[o][col][8 * c8]) = live ? __builtin_bit_cast(uint4, f) : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    bf16x8 qf[NS][NQ];
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int o = 0; o < NQ; ++o) qf[t][o] = *reinterpret_cast<const bf16x8*>(&qs[o][r16][64 * (t / 2) + 16 * kg + 8 * (t % 2)]);

    float m = -INFINITY, l = 0.0f;             // of the lane's head, exponents of two: m the same in all its lanes, l over this lane's keys
    f32x4 acc[NV];                             // O^T: element e of product j is d = NV (4 kg + e) + j of the lane's column
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float scale2 = a.scale * DEC8_LOG2E;

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
                for (int p = NQ - 1; p >= 0; --p) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][p], sc, 0, 0, 0);
            }
            const float f = scale2 * x.ks[hf];
#pragma unroll
            for (int e = 0; e < 4; ++e) s8[4 * hf + e] = (QP > 1 ? slot_sum<CS>(sc[e]) : sc[e]) * f;
        }
        if (32 * u + 32 > T) {
            asm volatile("; last unit");
#pragma unroll
            for (int i = 0; i < 8; ++i) s8[i] = 32 * u + 16 * (i / 4) + 4 * kg + i % 4 < T ? s8[i] : -INFINITY;
        }
        float bm = s8[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) bm = fmaxf(bm, s8[i]);
        const auto larger = [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); };
        bm = __uint_as_float(lane_step<32>(lane_step<16>(__float_as_uint(bm), larger), larger));
        // the reference follows the largest score once that is 2^8 times as likely: nothing is lost, and few units pay for it
        if (__any(bm > m + 8.0f)) {
            const float nm = fmaxf(m, bm);
            if (u != u0 + wave) {
                const float corr = __builtin_amdgcn_exp2f(m - nm);   // m > -inf: the wavefront's first unit has live keys
                l *= corr;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j][e] *= corr;
            }
            m = nm;
        }
        const float ref = m;
        float p8[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p8[i] = __builtin_amdgcn_exp2f(s8[i] - ref);             // 0 for a dead key
            l += p8[i];
        }
        bf16x8 pf[NP];
#pragma unroll
        for (int o = 0; o < NP; ++o) {
            const bool wanted = PPO == 1 || o * PPO + slot < PP;
            const float vs[2] = {wanted ? x.vs[0] : 0.0f, wanted ? x.vs[1] : 0.0f};
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = p8[i] * vs[i / 4];
            if constexpr (!O32) pf[o] = rounded_operand(y, PPO == 1 ? o == 1 : slot != 0);
            else pf[o] = PPO >= PP ? plane_operand<0, 2>(y, slot) : o == 0 ? plane_operand<0, PPO - 1>(y, slot) : o == 1 ? plane_operand<PPO, 2>(y, PPO + slot) : plane_operand<2, 2>(y, 2);
        }
#pragma unroll
        for (int c = 0; c < NW; ++c) {
            auto product = [&](auto bb) {
                constexpr int B = decltype(bb)::value;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (E4M3) {
                        // bytes B and B + 1 (B even) of two keys side by side, two of the four converted at a time
                        const uint32_t both = __builtin_amdgcn_perm(x.v[2 * i + 1][c], x.v[2 * i][c], B < 2 ? 0x05010400u : 0x07030602u);
                        w[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(both, 1.0f, B % 2 != 0));
                    } else {
                        w[i] = pack_bf16(code_value<E4M3, B>(x.v[2 * i][c]), code_value<E4M3, B>(x.v[2 * i + 1][c]));
                    }
                }
                const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                const int j = 4 * c + B;
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[p], acc[j], 0, 0, 0);
            };
            product(std::integral_constant<int, 0>{});
            product(std::integral_constant<int, 1>{});
            product(std::integral_constant<int, 2>{});
            product(std::integral_constant<int, 3>{});
        }
    };

    // Two units are on their way; behind the range's end, too, where they are fetched and not used (clamped to the sequence's
    // last).  Rows asked for against those needed: 16 ragged sequences of up to 2049 keys in four ranges 359 thousand for 248, 8
    // of 32768 keys in eight 4.43 million for 4.19.
    if (busy)
        for (int u = u0 + wave; u < u1; u += 2 * W) {
            compute(x0, u);
            if (u + W < u1) {
                load(x0, u + 2 * W);
                compute(x1, u + W);
                load(x1, u + 3 * W);
            }
        }

    // the wavefronts' partial softmaxes, merged in wavefront order
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < NV; j += 4) {
            const float4 v = make_float4(slot_sum<CS>(acc[j][e]), slot_sum<CS>(acc[j + 1][e]), slot_sum<CS>(acc[j + 2][e]), slot_sum<CS>(acc[j + 3][e]));
            if (slot == 0) *reinterpret_cast<float4*>(&part_o[wave][head][NV * (4 * kg + e) + j]) = v;
        }
    if (kg == 0 && slot == 0) { part_m[wave][head] = m; part_l[wave][head] = l; }
    __syncthreads();
    for (int i = tid; i < G * D; i += W * 64) {
        const int h = i / D, d = i % D;
        float gm = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) gm = fmaxf(gm, part_m[w][h]);
        const float ref = gm == -INFINITY ? 0.0f : gm;               // no key: every partial is empty
        float num = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = __builtin_amdgcn_exp2f(part_m[w][h] - ref);
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
                ml[0] = gm * DEC8_LN2;
                ml[1] = den;
            }
        }
    }
}

// ---- host side ----------------------------------------------------------------------

typedef void (*dec8_fn)(Dec8Args, AtomArgs);
typedef void (*append_fn)(Kv8AppendArgs, AtomArgs);

template <int D, int CS, int W>
static dec8_fn dec8_pick(bool e4m3, bool q32, bool o32)
{
    if (e4m3) return q32 ? (o32 ? attn_dec8_kernel<D, true, true, true, CS, W> : attn_dec8_kernel<D, true, true, false, CS, W>)
                         : (o32 ? attn_dec8_kernel<D, true, false, true, CS, W> : attn_dec8_kernel<D, true, false, false, CS, W>);
    return q32 ? (o32 ? attn_dec8_kernel<D, false, true, true, CS, W> : attn_dec8_kernel<D, false, true, false, CS, W>)
               : (o32 ? attn_dec8_kernel<D, false, false, true, CS, W> : attn_dec8_kernel<D, false, false, false, CS, W>);
}

template <int D, int W>
static dec8_fn dec8_group(const lithos_op_t& op)
{
    const bool e = op.flags & LITHOS_F_E4M3, q = op.flags & LITHOS_F_IN_F32, o = op.flags & LITHOS_F_OUT_F32;
    const int64_t G = op.dim[1] / op.dim[2];
    return G <= 4 ? dec8_pick<D, 4, W>(e, q, o) : G <= 8 ? dec8_pick<D, 8, W>(e, q, o) : dec8_pick<D, 16, W>(e, q, o);
}

// Four / eight wavefronts, us a pass with the merge: 16 ragged sequences, 8 heads of 128, whole (128 blocks) 19.9 / 18.9, 4 splits
// 16.9 / 22.1; 32 sequences of 512 keys, whole (256 blocks) 11.3 / 12.1; 8 of 32768, heads of 64, 4 splits 77 / 69, 8 splits 62 / 65.
static int dec8_waves(const lithos_op_t& op) { return op.dim[0] * op.dim[2] * std::max<int64_t>(1, op.dim[6]) >= 256 ? 4 : 8; }

static dec8_fn dec8_kernel(const lithos_op_t& op)
{
    if (dec8_waves(op) == 4) return op.dim[3] == 64 ? dec8_group<64, 4>(op) : dec8_group<128, 4>(op);
    return op.dim[3] == 64 ? dec8_group<64, 8>(op) : dec8_group<128, 8>(op);
}

// A workgroup per block for more than 16 tokens: 8192 bf16 tokens of 8 heads of 128 take 17.4 us with blocks of 32 positions,
// 21.5 with a wavefront per block, 64 tokens 5.3 and 8.5; one token 5.5 and 5.2.
static int append_waves(const lithos_op_t& op) { return op.dim[1] > 16 ? 4 : 1; }

template <int D, int WPU>
static append_fn append_pick(bool x32, bool e4m3)
{
    return x32 ? (e4m3 ? kv8_append_kernel<D, true, true, WPU> : kv8_append_kernel<D, true, false, WPU>)
               : (e4m3 ? kv8_append_kernel<D, false, true, WPU> : kv8_append_kernel<D, false, false, WPU>);
}

static append_fn append_kernel(const lithos_op_t& op)
{
    const bool e = op.flags & LITHOS_F_E4M3, x = op.flags & LITHOS_F_IN_F32;
    if (append_waves(op) == 4) return op.dim[3] == 64 ? append_pick<64, 4>(x, e) : append_pick<128, 4>(x, e);
    return op.dim[3] == 64 ? append_pick<64, 1>(x, e) : append_pick<128, 1>(x, e);
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
        if (op.flags & ~(LITHOS_F_IN_F32 | LITHOS_F_E4M3)) return fail(LITHOS_EINVAL, "kv8_append: takes IN_F32 and E4M3 only");
        if (!aligned16(op.in[0]) || !aligned16(op.in[1]) || !aligned16(op.out[0]) || !aligned16(op.out[1]))
            return fail(LITHOS_EINVAL, "kv8_append: keys, values and caches must be 16-byte aligned");
        if (!aligned_to(op.in[2], 4) || !aligned_to(op.in[3], 4)) return fail(LITHOS_EINVAL, "kv8_append: misaligned positions or scales");
        if (op.ld[0] < n_kv * d || op.ld[0] % (x32 ? 4 : 8)) return fail(LITHOS_EINVAL, "kv8_append: row stride %lld is smaller than n_kv*d or breaks the 16-byte alignment of rows", (long long)op.ld[0]);
        const int64_t units = 2 * batch * touched_blocks(op) * n_kv;
        const int64_t groups = append_waves(op) == 4 ? units : (units + 3) / 4;
        if (groups > 0x7fffffff) return fail(LITHOS_EINVAL, "kv8_append: too many workgroups");
        plan->grid = {(uint32_t)groups, 1, 1};
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
    if (op.flags & ~(LITHOS_F_IN_F32 | LITHOS_F_OUT_F32 | LITHOS_F_E4M3)) return fail(LITHOS_EINVAL, "attn_dec8: takes IN_F32, OUT_F32 and E4M3 only");
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
    plan->threads = dec8_waves(op) * 64;
    plan->wg_per_cu = cached_occupancy((const void*)dec8_kernel(op), (int)plan->threads, 1);
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
    a.keys = (int)op.dim[4]; a.splits = op.dim[6] > 0 ? (int)op.dim[6] : 1;
    a.nblk = (int)ceil_div(op.dim[5], op.dim[7]);
    a.seq = op.dim[5] * op.dim[2] * op.dim[3];
    // floor(h / d) = floor(h ceil(2^32 / d) / 2^32) for h < 2^26, d <= 64: the rounding adds less than h d / 2^32 / d <= 1 / d
    a.blk_magic = op.dim[7] == 16 ? 0u : (uint32_t)ceil_div(1ll << 32, op.dim[7] / 16);
    LITHOS_HIP(launch_kernel(dec8_kernel(op), grid, block, s, a, atom));
    return LITHOS_OK;
}

// Key ranges per (sequence, key/value head).  One CU fetches some 27 bytes a nanosecond, and a launch with its merge costs
// about 4 us: up to 128 KB a workgroup stays alone (8 heads of 128, whole / 2 / 4 / 8 splits, us a pass: 300 keys 7.3, 10.8, 10.0,
// 9.7, 512 keys 9.3, 11.3, 10.0, 9.5, 1024 keys 12.6, 13.7, 11.2, 9.9).  Beyond, ranges of at least 128 keys, a unit for each
// of four wavefronts, as many as the chip holds at a time: two workgroups of four wavefronts on a CU (heads of 64: four), or,
// where that would be more than eight ranges to merge, one of eight (16 ragged sequences 2, 4, 8 splits 18.0, 16.9, 20.5).
int kv8_split_hint(const lithos_op_t& op, int n_cus)
{
    const int64_t bytes = 2 * op.dim[3] * op.dim[4], pairs = op.dim[0] * op.dim[2], per_cu = op.dim[3] == 64 ? 4 : 2;
    if (bytes <= 128 * 1024) return 1;
    int64_t s = per_cu * n_cus / pairs;
    if (s > 8) s = std::max<int64_t>(8, per_cu / 2 * n_cus / pairs);
    return (int)std::max<int64_t>(1, std::min({s, ceil_div(op.dim[4], 128), (int64_t)LITHOS_ATTN_MAX_SPLITS}));
}

} // namespace lithos
