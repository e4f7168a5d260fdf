// Log probabilities of given tokens, entropy, log-sum-exp and the most likely tokens of rows of logits, and the gradient.
//
// With z = c x (c the scale, an inverse temperature), per row:
//   lse = log sum_i exp z_i,   logprob = z_t - lse,   H = lse - sum_i p_i z_i,   p_i = exp(z_i - lse),
//   and the `top` largest x, equal ones by the lower index.
// One pass: with m the largest x so far, d_i = c (x_i - m), l = sum exp d_i and t = sum exp(d_i) d_i,
//   lse = c m + log l,   H = log l - t / l;   when m rises by r (in units of d): t <- f (t - l r), l <- f l, f = exp(-r).
// Each lane keeps (m, l, t) of its own elements; lanes, wavefronts and splits are joined in a fixed order.
//
// The most likely tokens: a wavefront keeps a list of up to `top` keys (value, index) in LDS.  Elements above its
// smallest value are rare once it is full; they are gathered behind it and the list is chosen anew when 64 wait.  The
// first tile fills the list: the top-th of the 64 lanes' largest keys is a bound below which nothing can be chosen.
// Bound by the bytes of the logits, read once.
#include "common.hpp"
#include <math.h>
#include <algorithm>

namespace lithos {

struct LogprobArgs {
    const void* x;
    const int32_t* targets;     // nullptr: no given tokens
    float* stats;               // per row: logprob, entropy, lse, then the top's log probabilities
    int32_t* ids;
    float* ws;
    int64_t ldx, lds, ldi;
    int rows, vocab, top, splits;
    float scale;
};

constexpr int LP_TOP = LITHOS_LOGPROBS_MAX_TOP, LP_WAIT = 128;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// larger key = larger value, then lower index; -0 is 0
__device__ __forceinline__ uint64_t top_key(float x, uint32_t idx)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return ((uint64_t)(b ^ (b & 0x80000000u ? 0xffffffffu : 0x80000000u)) << 32) | (0xffffffffu - idx);
}
__device__ __forceinline__ float key_value(uint64_t k)
{
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - (uint32_t)k; }

// sums of a softmax over some elements, d in powers of two
struct Soft { float m, l, t; };

__device__ __forceinline__ Soft soft_join(const Soft& a, const Soft& b, float c2)
{
    Soft r;
    r.m = fmaxf(a.m, b.m);
    const float ref = r.m == -INFINITY ? 0.0f : r.m;
    // an empty side (m = -inf, l = t = 0) adds nothing; its distance must not become infinity times zero
    const float ra = fmaxf((a.m - ref) * c2, -300.0f), rb = fmaxf((b.m - ref) * c2, -300.0f);
    const float fa = __builtin_amdgcn_exp2f(ra), fb = __builtin_amdgcn_exp2f(rb);
    r.l = fa * a.l + fb * b.l;
    r.t = fa * fmaf(ra, a.l, a.t) + fb * fmaf(rb, b.l, b.t);
    return r;
}

__device__ __forceinline__ Soft soft_wave(Soft s, float c2)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const Soft b = {__shfl_xor(s.m, o), __shfl_xor(s.l, o), __shfl_xor(s.t, o)};
        s = soft_join(s, b, c2);
    }
    return s;
}

// The k largest of n keys (n <= 64 * PER), sorted, at out[0 .. min(k, n)); keys are distinct.  One wavefront.
template <int PER>
__device__ __forceinline__ void choose_top(const uint64_t* keys, int n, int k, uint64_t* out, int lane)
{
    uint64_t mine[PER];
    int above[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) { mine[i] = i * 64 + lane < n ? keys[i * 64 + lane] : 0; above[i] = 0; }
    for (int j = 0; j < n; ++j) {
        const uint64_t o = keys[j];
#pragma unroll
        for (int i = 0; i < PER; ++i) above[i] += o > mine[i];
    }
    wave_lds_sync();                             // `out` may overlap `keys`
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < n && above[i] < k) out[above[i]] = mine[i];
    wave_lds_sync();
}

// what is written of a row
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Soft& s, float logit, bool given, const uint64_t* top, int lane)
{
    const float ln = logf(s.l);
    const bool none = s.m == -INFINITY && s.l == 0.0f;          // no token is allowed
    float* st = a.stats + row * a.lds;
    if (lane == 0) {
        st[0] = !given ? 0.0f : logit == -INFINITY ? -INFINITY : a.scale * (logit - s.m) - ln;
        st[1] = none ? 0.0f : ln - s.t * LN2 / s.l;
        st[2] = none ? -INFINITY : fmaf(a.scale, s.m, ln);
    }
    if (lane < a.top) {
        const float x = key_value(top[lane]);
        st[3 + lane] = x == -INFINITY ? -INFINITY : a.scale * (x - s.m) - ln;
        a.ids[row * a.ldi + lane] = (int32_t)key_index(top[lane]);
    }
}

template <bool X32>
__device__ __forceinline__ float logit_at(const LogprobArgs& a, int64_t row, int64_t i)
{
    if constexpr (X32) return reinterpret_cast<const float*>(a.x)[row * a.ldx + i];
    else return bf16_to_f32(reinterpret_cast<const uint16_t*>(a.x)[row * a.ldx + i]);
}

// the given token of a row, -1 if it has none
__device__ __forceinline__ int given_token(const LogprobArgs& a, int64_t row)
{
    const int t = a.targets ? a.targets[row] : -1;
    return (uint32_t)t < (uint32_t)a.vocab ? t : -1;
}

typedef float f32x4_b4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_b2 __attribute__((ext_vector_type(4), aligned(2)));

// Logical block = (row, split).  The split's elements are tiles of 1024 which its four wavefronts take in turn; a lane
// owns 16 of a tile, in runs of 4 (fp32) or 8 (bf16).
template <bool X32>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobArgs a, AtomArgs atom)
{
    constexpr int RUN = X32 ? 4 : 8, TILE = 1024;
    __shared__ uint64_t keys[4][LP_TOP + LP_WAIT];
    __shared__ Soft softs[4];
    __shared__ int counts[4];

    const uint32_t L = atom_logical_block(atom);
    const int64_t row = L / a.splits;
    const int sp = L % a.splits;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = (a.vocab + TILE - 1) / TILE;
    const int t0 = (int)((int64_t)sp * tiles / a.splits), t1 = (int)((int64_t)(sp + 1) * tiles / a.splits);
    const float c2 = a.scale * LOG2E;
    const int K = a.top;

    const char* const xrow = reinterpret_cast<const char*>(a.x) + row * a.ldx * (X32 ? 4 : 2);
    auto index = [&](int tile, int e) { return tile * TILE + (e / RUN) * 64 * RUN + lane * RUN + e % RUN; };
    auto load = [&](int tile, float (&x)[16]) {
        if ((tile + 1) * TILE <= a.vocab) {
            if constexpr (X32) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4_b4 v = *reinterpret_cast<const f32x4_b4*>(xrow + (int64_t)index(tile, 4 * q) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * q + e] = v[e];
                }
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const u32x4_b2 v = *reinterpret_cast<const u32x4_b2*>(xrow + (int64_t)index(tile, 8 * q) * 2);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { x[8 * q + 2 * e] = __uint_as_float(v[e] << 16); x[8 * q + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = index(tile, e);
                x[e] = i < a.vocab ? logit_at<X32>(a, row, i) : -INFINITY;
            }
        }
    };

    Soft s = {-INFINITY, 0.0f, 0.0f};
    uint64_t* const list = keys[wave];
    int have = 0, wait = 0;                       // keys chosen, keys waiting behind place LP_TOP
    uint64_t least_key = 0;                       // smallest key chosen, once K are, and its value
    float least = -INFINITY;
    auto choose = [&]() {
        // chosen keys first, waiting ones behind them without a gap
        uint64_t moved[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) moved[i] = i * 64 + lane < wait ? list[LP_TOP + i * 64 + lane] : 0;
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < 2; ++i) if (i * 64 + lane < wait) list[have + i * 64 + lane] = moved[i];
        wave_lds_sync();
        choose_top<3>(list, have + wait, K, list, lane);
        have = min(K, have + wait);
        wait = 0;
        if (have == K) { least_key = list[K - 1]; least = key_value(least_key); }
    };
    auto gather = [&](bool mine, uint64_t key) {
        const uint64_t all = __ballot(mine);
        if (all == 0) return;
        if (mine) list[LP_TOP + wait + __popcll(all & ((1ull << lane) - 1))] = key;
        wait += __popcll(all);
        wave_lds_sync();
        if (wait > LP_WAIT - 64) choose();
    };

    bool first = true;
    for (int tile = t0 + wave; tile < t1; tile += 4) {
        float x[16];
        load(tile, x);
        float mt = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, x[e]);
        if (__any(mt > s.m)) {
            const float nm = fmaxf(s.m, mt), ref = nm == -INFINITY ? 0.0f : nm;
            const float r = fmaxf((s.m - ref) * c2, -300.0f), f = __builtin_amdgcn_exp2f(r);
            s.t = f * fmaf(r, s.l, s.t);
            s.l *= f;
            s.m = nm;
        }
        const float ref = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            // the difference first: products of masks of the type's lowest value overflow
            const float d = (x[e] - ref) * c2, p = __builtin_amdgcn_exp2f(d);
            s.l += p;
            s.t = fmaf(p, fmaxf(d, -300.0f), s.t);            // 0, not infinity times 0, for a forbidden token
        }
        if (K == 0) continue;
        if (first) {
            first = false;
            uint64_t best = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = index(tile, e);
                const uint64_t k = top_key(x[e], i);
                if (i < a.vocab && k > best) best = k;
            }
            int above = 0;
            for (int j = 0; j < 64; ++j) above += __shfl(best, j) > best;
            // the K-th largest of the lanes' best keys (0, of a lane without elements, if there are not as many)
            const uint64_t at = __ballot(above == K - 1 && best != 0);
            const uint64_t bound = at ? __shfl(best, __ffsll((unsigned long long)at) - 1) : 1;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = index(tile, e);
                const uint64_t k = top_key(x[e], i);
                gather(i < a.vocab && k >= bound, k);
            }
            choose();
        } else if (have < K || __any(mt > least)) {           // an equal value of a later tile has a higher index
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = index(tile, e);
                const uint64_t k = top_key(x[e], i);
                gather(i < a.vocab && k > least_key, k);
            }
        }
    }
    if (wait) choose();
    s = soft_wave(s, c2);
    if (lane == 0) { softs[wave] = s; counts[wave] = have; }
    __syncthreads();
    if (wave != 0) return;

    s = softs[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) s = soft_join(s, softs[w], c2);
    // the four lists, one after another, in the first two wavefronts' room
    uint64_t* const all = keys[0];
    int n = counts[0];
    for (int w = 1; w < 4; ++w) {
        const uint64_t k = lane < counts[w] ? keys[w][lane] : 0;
        wave_lds_sync();
        if (lane < counts[w]) all[n + lane] = k;
        wave_lds_sync();
        n += counts[w];
    }
    choose_top<2>(all, n, K, all, lane);
    n = min(n, K);
    if (a.splits == 1) {
        const int t = given_token(a, row);
        write_row(a, row, s, t >= 0 ? logit_at<X32>(a, row, t) : 0.0f, t >= 0, all, lane);
    } else {
        float* w = a.ws + ((int64_t)row * a.splits + sp) * (4 + 2 * K);
        if (lane == 0) { w[0] = s.m; w[1] = s.l; w[2] = s.t; w[3] = (float)n; }
        if (lane < n) reinterpret_cast<uint2*>(w + 4)[lane] = make_uint2((uint32_t)all[lane], (uint32_t)(all[lane] >> 32));
    }
}

// Joins the splits of a row, in split order.  One workgroup of one wavefront's work per row; four rows per workgroup.
template <bool X32>
__global__ __launch_bounds__(256) void logprobs_merge_kernel(LogprobArgs a, AtomArgs atom)
{
    __shared__ uint64_t keys[4][3 * 64];
    const uint32_t L = atom_logical_block(atom);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)L * 4 + wave;
    if (row >= a.rows) return;
    const float c2 = a.scale * LOG2E;
    const int K = a.top;
    Soft s = {-INFINITY, 0.0f, 0.0f};
    uint64_t* const list = keys[wave];
    int n = 0;
    for (int sp = 0; sp < a.splits; ++sp) {
        const float* w = a.ws + (row * a.splits + sp) * (4 + 2 * K);
        s = soft_join(s, Soft{w[0], w[1], w[2]}, c2);
        const int more = (int)w[3];
        if (lane < more) {
            const uint2 k = reinterpret_cast<const uint2*>(w + 4)[lane];
            list[n + lane] = ((uint64_t)k.y << 32) | k.x;
        }
        n += more;
        wave_lds_sync();
        if (n > 3 * 64 - LP_TOP) { choose_top<3>(list, n, K, list, lane); n = K; }
    }
    choose_top<3>(list, n, K, list, lane);
    const int t = given_token(a, row);
    write_row(a, row, s, t >= 0 ? logit_at<X32>(a, row, t) : 0.0f, t >= 0, list, lane);
}

// ---- gradient ------------------------------------------------------------------------
//   dx_i = c (g_lp (1[i = t] - p_i) - g_H p_i (log p_i + H)),   log p_i = c x_i - lse
// with lse and H from the forward pass.  A forbidden token (x = -inf) and a row without allowed ones get 0.
struct LogprobGradArgs {
    const void* x;
    const int32_t* targets;
    const float* stats;
    const float* g_lp;
    const float* g_ent;         // nullptr: 0
    void* dx;
    int64_t ldx, lds, ldd;
    int rows, vocab, per_row;   // blocks of a row
    float scale;
};

template <bool X32, bool D32>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(LogprobGradArgs a, AtomArgs atom)
{
    constexpr int RUN = 8, STEP = 256 * RUN;
    const uint32_t L = atom_logical_block(atom);
    const int64_t row = L / a.per_row;
    const int i0 = (int)(L % a.per_row) * STEP + threadIdx.x * RUN;
    if (i0 >= a.vocab) return;
    const float H = a.stats[row * a.lds + 1], lse = a.stats[row * a.lds + 2];
    const int t = a.targets ? a.targets[row] : -1;
    const float g = (uint32_t)t < (uint32_t)a.vocab && a.g_lp ? a.g_lp[row] : 0.0f, ge = a.g_ent ? a.g_ent[row] : 0.0f;
    const float c = a.scale;
    const int n = min(RUN, a.vocab - i0);
    const char* xp = reinterpret_cast<const char*>(a.x) + (row * a.ldx + i0) * (X32 ? 4 : 2);
    float x[RUN], d[RUN];
    if (n == RUN) {
        if constexpr (X32) {
            const f32x4_b4 u = *reinterpret_cast<const f32x4_b4*>(xp), v = *reinterpret_cast<const f32x4_b4*>(xp + 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = u[e]; x[4 + e] = v[e]; }
        } else {
            const u32x4_b2 v = *reinterpret_cast<const u32x4_b2*>(xp);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(v[e] << 16); x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
        }
    } else {
#pragma unroll
        for (int e = 0; e < RUN; ++e) {
            if constexpr (X32) x[e] = e < n ? reinterpret_cast<const float*>(xp)[e] : 0.0f;
            else x[e] = e < n ? bf16_to_f32(reinterpret_cast<const uint16_t*>(xp)[e]) : 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < RUN; ++e) {
        const float lp = fmaf(c, x[e], -lse), p = __builtin_amdgcn_exp2f(lp * LOG2E);
        float dz = -p * fmaf(ge, lp + H, g);
        if (i0 + e == t) dz += g;
        if (x[e] == -INFINITY) dz = 0.0f;
        d[e] = c * dz;
    }
    char* dp = reinterpret_cast<char*>(a.dx) + (row * a.ldd + i0) * (D32 ? 4 : 2);
    if (n == RUN) {
        if constexpr (D32) {
            *reinterpret_cast<f32x4_b4*>(dp) = f32x4_b4{d[0], d[1], d[2], d[3]};
            *reinterpret_cast<f32x4_b4*>(dp + 16) = f32x4_b4{d[4], d[5], d[6], d[7]};
        } else {
            *reinterpret_cast<u32x4_b2*>(dp) = u32x4_b2{pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < RUN; ++e)
            if (e < n) {
                if constexpr (D32) reinterpret_cast<float*>(dp)[e] = d[e];
                else reinterpret_cast<uint16_t*>(dp)[e] = f32_to_bf16(d[e]);
            }
    }
}

// ---- host side ----------------------------------------------------------------------

typedef void (*lp_fn)(LogprobArgs, AtomArgs);
typedef void (*lp_grad_fn)(LogprobGradArgs, AtomArgs);

static lp_fn lp_kernel(const lithos_op_t& op)
{
    const bool x32 = op.flags & LITHOS_F_IN_F32;
    if (op.kind == LITHOS_OP_LOGPROBS) return x32 ? logprobs_kernel<true> : logprobs_kernel<false>;
    return x32 ? logprobs_merge_kernel<true> : logprobs_merge_kernel<false>;
}

static lp_grad_fn lp_grad_kernel(const lithos_op_t& op)
{
    if (op.flags & LITHOS_F_IN_F32) return op.flags & LITHOS_F_OUT_F32 ? logprobs_grad_kernel<true, true> : logprobs_grad_kernel<true, false>;
    return op.flags & LITHOS_F_OUT_F32 ? logprobs_grad_kernel<false, true> : logprobs_grad_kernel<false, false>;
}

int logprobs_plan(const lithos_op_t& op, OpPlan* plan)
{
    // dim = rows, vocab, top, splits; ld = row strides of logits, stats, ids (gradient: logits, stats, dlogits)
    const int64_t rows = op.dim[0], vocab = op.dim[1], top = op.dim[2];
    const int64_t splits = op.dim[3] > 0 ? op.dim[3] : 1;
    const bool grad = op.kind == LITHOS_OP_LOGPROBS_GRAD, x32 = op.flags & LITHOS_F_IN_F32;
    if (rows <= 0 || vocab <= 0 || rows > (1ll << 31) - 1 || vocab > (1ll << 30))
        return fail(LITHOS_EINVAL, "logprobs: rows and vocabulary must be positive (got %lld, %lld)", (long long)rows, (long long)vocab);
    if (!(op.fparam[0] > 0.0f) || !(op.fparam[0] < INFINITY)) return fail(LITHOS_EINVAL, "logprobs: the scale (fparam0) must be positive and finite");
    if (op.ld[0] < vocab) return fail(LITHOS_EINVAL, "logprobs: row stride of the logits smaller than the vocabulary");
    if (!op.in[0] || reinterpret_cast<uintptr_t>(op.in[0]) % (x32 ? 4 : 2)) return fail(LITHOS_EINVAL, "logprobs: null or misaligned logits");
    if (!aligned_to(op.in[1], 4)) return fail(LITHOS_EINVAL, "logprobs: misaligned tokens");
    plan->threads = 256;
    plan->variant = 0;
    plan->wg_per_cu = 8;
    uint64_t blocks;
    if (grad) {
        if (!op.in[2] || op.ld[1] < 3) return fail(LITHOS_EINVAL, "logprobs_grad: needs the forward pass's statistics in in[2], a row stride of at least 3");
        if (op.in[3] && !op.in[1]) return fail(LITHOS_EINVAL, "logprobs_grad: a gradient of log probabilities (in[3]) needs their tokens in in[1]");
        if (!aligned_to(op.in[2], 4) || !aligned_to(op.in[3], 4) || !aligned_to(op.in[4], 4)) return fail(LITHOS_EINVAL, "logprobs_grad: misaligned statistics or gradients");
        if (!op.out[0] || reinterpret_cast<uintptr_t>(op.out[0]) % (op.flags & LITHOS_F_OUT_F32 ? 4 : 2) || op.ld[2] < vocab)
            return fail(LITHOS_EINVAL, "logprobs_grad: null or misaligned output, or a row stride smaller than the vocabulary");
        if (op.in[0] == op.out[0] && (x32 != (bool)(op.flags & LITHOS_F_OUT_F32) || op.ld[0] != op.ld[2]))
            return fail(LITHOS_EINVAL, "logprobs_grad: in place needs logits and gradient of one type and stride");
        blocks = (uint64_t)rows * ((vocab + 2047) / 2048);
    } else {
        if (top < 0 || top > LITHOS_LOGPROBS_MAX_TOP || top > vocab) return fail(LITHOS_EINVAL, "logprobs: top %lld outside 0 .. min(vocabulary, %d)", (long long)top, LITHOS_LOGPROBS_MAX_TOP);
        if (!aligned_to(op.out[0], 4) || !aligned_to(op.out[1], 4)) return fail(LITHOS_EINVAL, "logprobs: misaligned statistics or token output");
        if (!op.out[0] || op.ld[1] < 3 + top) return fail(LITHOS_EINVAL, "logprobs: null statistics, or a row stride smaller than 3 + top");
        if (top && (!op.out[1] || op.ld[2] < top)) return fail(LITHOS_EINVAL, "logprobs: null token output, or a row stride smaller than top");
        if (splits > LITHOS_LOGPROBS_MAX_SPLITS) return fail(LITHOS_EINVAL, "logprobs: splits %lld above %d", (long long)splits, LITHOS_LOGPROBS_MAX_SPLITS);
        const bool merge = op.kind == LITHOS_OP_LOGPROBS_MERGE;
        if ((merge || splits > 1) && (!op.in[2] || !aligned16(op.in[2]))) return fail(LITHOS_EINVAL, "logprobs: a split launch and its merge need a 16-byte aligned workspace in in[2]");
        blocks = merge ? (uint64_t)(rows + 3) / 4 : (uint64_t)rows * splits;
    }
    if (blocks > 0x7fffffffull) return fail(LITHOS_EINVAL, "logprobs: too many workgroups");
    plan->grid = {(uint32_t)blocks, 1, 1};
    plan->total = (uint32_t)blocks;
    plan->wg_per_cu = cached_occupancy(grad ? (const void*)lp_grad_kernel(op) : (const void*)lp_kernel(op), 256, 4);
    return LITHOS_OK;
}

int logprobs_launch(const lithos_op_t& op, const OpPlan& plan, const AtomArgs& atom, hipStream_t s)
{
    const dim3 grid(LITHOS_ATOM_LAUNCH_BLOCKS(atom)), block(plan.threads);
    if (op.kind == LITHOS_OP_LOGPROBS_GRAD) {
        LogprobGradArgs a{};
        a.x = op.in[0]; a.targets = (const int32_t*)op.in[1]; a.stats = (const float*)op.in[2];
        a.g_lp = (const float*)op.in[3]; a.g_ent = (const float*)op.in[4];
        a.dx = op.out[0];
        a.ldx = op.ld[0]; a.lds = op.ld[1]; a.ldd = op.ld[2];
        a.rows = (int)op.dim[0]; a.vocab = (int)op.dim[1]; a.per_row = (a.vocab + 2047) / 2048;
        a.scale = op.fparam[0];
        LITHOS_HIP(launch_kernel(lp_grad_kernel(op), grid, block, s, a, atom));
        return LITHOS_OK;
    }
    LogprobArgs a{};
    a.x = op.in[0]; a.targets = (const int32_t*)op.in[1]; a.ws = (float*)const_cast<void*>(op.in[2]);
    a.stats = (float*)op.out[0]; a.ids = (int32_t*)op.out[1];
    a.ldx = op.ld[0]; a.lds = op.ld[1]; a.ldi = op.ld[2];
    a.rows = (int)op.dim[0]; a.vocab = (int)op.dim[1]; a.top = (int)op.dim[2]; a.splits = op.dim[3] > 0 ? (int)op.dim[3] : 1;
    a.scale = op.fparam[0];
    LITHOS_HIP(launch_kernel(lp_kernel(op), grid, block, s, a, atom));
    return LITHOS_OK;
}

// Two workgroups per CU of the target, each with a tile of 1024 for every one of its four wavefronts.
int logprobs_split_hint(const lithos_op_t& op, int n_cus)
{
    const int64_t quads = (op.dim[1] + 4095) / 4096, want = (2ll * n_cus + op.dim[0] - 1) / op.dim[0];
    return (int)std::max<int64_t>(1, std::min({quads, want, (int64_t)LITHOS_LOGPROBS_MAX_SPLITS}));
}

} // namespace lithos
