// Log probabilities of given tokens, entropy, log-sum-exp and the most likely tokens of rows of logits, and the gradient.
//
// With z = c x (c the scale, an inverse temperature), per row:
//   lse = log sum_i exp z_i,   logprob = z_t - lse,   H = lse - sum_i p_i z_i,   p_i = exp(z_i - lse),
//   and the `top` largest x, equal ones by the lower index.
// One pass: with m the largest x so far, d_i = c (x_i - m), l = sum exp d_i and t = sum exp(d_i) d_i,
//   lse = c m + log l,   H = log l - t / l;   when m rises by r (in units of d): t <- f (t - l r), l <- f l, f = exp(-r).
// Each lane keeps (m, l, t) of its own elements; lanes, wavefronts and splits are joined in a fixed order.
//
// The most likely tokens (stream): every lane notes the largest of its elements in each of up to eight stretches.  If m of the
// four wavefronts have j lanes each, m j >= top, whose largest element reaches a bound, so do `top` elements, all of them in
// the few stretches whose largest does; the bound is the best for m = 4, 2 and 1.  The elements of these stretches are read a
// second time; those that reach the bound find their places by counting larger ones.  (A list kept during the pass cost more:
// 2048 rows of 131072 bf16 took 132 us with top = 5 and 171 with 32.)
// Bound by the bytes of the logits, read once: 2048 rows of 131072 bf16 take 111 us with top = 5, 4.8 TB/s, 105 without.  A CU
// alone does 8 tokens a ns, which bounds few rows.
#include "common.hpp"
#include <float.h>
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

constexpr int LP_TOP = LITHOS_LOGPROBS_MAX_TOP, LP_ROOM = 2048, LP_PAD = 32, LP_SEG = 8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_b4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_b2 __attribute__((ext_vector_type(4), aligned(2)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// larger number = larger value; -0 is 0
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b & 0x80000000u ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

// larger key = larger value, then lower index
__device__ __forceinline__ uint64_t top_key(float x, uint32_t idx) { return ((uint64_t)ordered(x) << 32) | (0xffffffffu - idx); }
__device__ __forceinline__ float key_value(uint64_t k) { return value_of((uint32_t)(k >> 32)); }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - (uint32_t)k; }

// sums of a softmax over some elements, d in powers of two
struct Soft { float m, l, t; };

template <int N>
__device__ __forceinline__ float group_max(float x)
{
    return __uint_as_float(lane_group<N>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int N>
__device__ __forceinline__ float group_sum(float x)
{
    return __uint_as_float(lane_group<N>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// The least of the maxima of the lanes' residue classes modulo `groups`, a power of two.
__device__ __forceinline__ uint32_t least_of_groups(uint32_t x, int groups)
{
    auto join = [&](int stride) { return [=](uint32_t a, uint32_t b) { return stride >= groups ? max(a, b) : min(a, b); }; };
    x = lane_step<32>(x, join(32));
    x = lane_step<16>(x, join(16));
    x = join(8)(x, lane_from<0x128>(x));          // row_ror: modulo 16 the neighbour at that distance
    x = join(4)(x, lane_from<0x124>(x));
    x = join(2)(x, lane_from<0x122>(x));
    return join(1)(x, lane_from<0x121>(x));
}

__device__ __forceinline__ int power_of_two_from(int n) { return n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// the sums of N lanes, referred to the largest of their references
template <int N>
__device__ __forceinline__ Soft soft_all(const Soft& s, float c2)
{
    Soft r;
    r.m = group_max<N>(s.m);
    // an empty side (m = -inf, l = t = 0) adds nothing; its distance must not become infinity times zero
    const float d = fmaxf((s.m - (r.m == -INFINITY ? 0.0f : r.m)) * c2, -300.0f), f = __builtin_amdgcn_exp2f(d);
    r.l = group_sum<N>(f * s.l);
    r.t = group_sum<N>(f * fmaf(d, s.l, s.t));
    return r;
}

// the sums of W wavefronts, the same in all lanes
template <int W>
__device__ __forceinline__ Soft soft_of_waves(const Soft* softs, int lane, float c2)
{
    const Soft s = soft_all<16>(lane < W ? softs[lane] : Soft{-INFINITY, 0.0f, 0.0f}, c2);
    auto first = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    return Soft{first(s.m), first(s.l), first(s.t)};
}

// The k largest of n distinct keys in LDS, sorted, to `out`: a key's place is the number of larger ones.  By the whole
// workgroup of NT, up to eight neighbouring threads to a key; behind the keys there is room for LP_PAD more.  The caller puts
// barriers around it.
template <int NT>
__device__ __forceinline__ void choose_top(uint64_t* keys, int n, int k, uint64_t* out)
{
    if (threadIdx.x < LP_PAD) keys[n + threadIdx.x] = 0;                          // larger than none
    __syncthreads();
    const int share = n > NT / 2 ? 0 : n > NT / 4 ? 1 : n > NT / 8 ? 2 : 3;       // log2 of the threads to a key
    const int part = threadIdx.x & ((1 << share) - 1), stride = 4 << share;
    for (int i0 = 0; i0 < n; i0 += NT >> share) {
        const int i = i0 + (threadIdx.x >> share);
        const uint64_t mine = keys[min(i, n - 1)];
        uint32_t above = 0;
#pragma unroll 2
        for (int o = 4 * part; o < n; o += stride)
#pragma unroll
            for (int u = 0; u < 4; ++u) above += keys[o + u] > mine;
        const auto add = [](uint32_t a, uint32_t b) { return a + b; };
        if (share >= 1) above = lane_step<1>(above, add);
        if (share >= 2) above = lane_step<2>(above, add);
        if (share >= 3) above = lane_step<4>(above, add);
        if (i < n && part == 0 && above < (uint32_t)k) out[above] = mine;
    }
}

// what is written of a row
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Soft& s, float logit, bool given, const uint64_t* top, int lane)
{
    const float ln = logf(s.l);
    const bool none = s.m == -INFINITY && s.l == 0.0f;          // no token is allowed
    const bool broken = s.l != s.l;                             // a NaN or +infinity in the row: that decides before a -infinity does
    float* st = a.stats + row * a.lds;
    if (lane == 0) {
        st[0] = !given ? 0.0f : logit == -INFINITY && !broken ? -INFINITY : a.scale * (logit - s.m) - ln;
        st[1] = none ? 0.0f : ln - s.t * LN2 / s.l;
        st[2] = none ? -INFINITY : fmaf(a.scale, s.m, ln);
    }
    if (lane < a.top) {
        const float x = key_value(top[lane]);
        st[3 + lane] = x == -INFINITY && !broken ? -INFINITY : a.scale * (x - s.m) - ln;
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


// A row's elements lie in tiles of 1024.  A lane owns 16 of a tile, in runs of 4 (fp32) or 8 (bf16).
constexpr int LP_TILE = 1024;
template <bool X32>
struct LogitRow {
    static constexpr int RUN = X32 ? 4 : 8;
    const char* x;
    int vocab;

    __device__ __forceinline__ bool whole(int tile) const { return (tile + 1) * LP_TILE <= vocab; }
    // element e of lane l; the last, partial tile is dealt out one element after another, so that every lane has some
    __device__ __forceinline__ int index(int tile, int l, int e) const { return tile * LP_TILE + (whole(tile) ? (e / RUN) * 64 * RUN + l * RUN + e % RUN : e * 64 + l); }
    // elements RUN q .. RUN q + RUN - 1 of lane l as four dwords
    __device__ __forceinline__ u32x4 load_whole(int tile, int l, int q) const
    {
        return u32x4(*reinterpret_cast<const u32x4_b2*>(x + (int64_t)(tile * LP_TILE + q * 64 * RUN + l * RUN) * (X32 ? 4 : 2)));
    }
    __device__ __forceinline__ u32x4 load_partial(int tile, int l, int q) const       // what lies beyond the row is -infinity
    {
        uint32_t one[RUN];
#pragma unroll
        for (int e = 0; e < RUN; ++e) {
            const int at = min(tile * LP_TILE + (RUN * q + e) * 64 + l, vocab - 1);
            if constexpr (X32) one[e] = reinterpret_cast<const uint32_t*>(x)[at];
            else one[e] = reinterpret_cast<const uint16_t*>(x)[at];
        }
#pragma unroll
        for (int e = 0; e < RUN; ++e) if (tile * LP_TILE + (RUN * q + e) * 64 + l >= vocab) one[e] = X32 ? 0xff800000u : 0xff80u;
        u32x4 v;
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = X32 ? one[d] : one[(2 * d) % RUN] | (one[(2 * d + 1) % RUN] << 16);
        return v;
    }
    __device__ __forceinline__ u32x4 load(int tile, int l, int q) const { return whole(tile) ? load_whole(tile, l, q) : load_partial(tile, l, q); }
    __device__ __forceinline__ void unpack(const u32x4& v, float* f) const
    {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if constexpr (X32) f[d] = __uint_as_float(v[d]);
            else { f[2 * d] = __uint_as_float(v[d] << 16); f[2 * d + 1] = __uint_as_float(v[d] & 0xffff0000u); }
        }
    }
};

// the row's or the split's n chosen keys, by the whole workgroup: to the workspace, or made K of them (rows with NaN: any token)
__device__ __forceinline__ void save_top(const LogprobArgs& a, int64_t row, int sp, int n, uint64_t* chosen)
{
    const int tid = threadIdx.x, K = a.top;
    if (a.splits == 1) {
        if (tid >= n && tid < K) chosen[tid] = top_key(-INFINITY, tid);
    } else if (tid < 64) {
        float* w = a.ws + (row * a.splits + sp) * (4 + 2 * K);
        if (tid == 0) w[3] = (float)n;
        if (tid < n) reinterpret_cast<uint2*>(w + 4)[tid] = make_uint2((uint32_t)chosen[tid], (uint32_t)(chosen[tid] >> 32));
    }
}

// the rest of the results, by one wavefront, the first
__device__ __forceinline__ void save_sums(const LogprobArgs& a, int64_t row, int sp, const Soft& s, int token, float logit, const uint64_t* chosen, int lane)
{
    if (a.splits == 1) {
        wave_lds_sync();
        write_row(a, row, s, logit, token >= 0, chosen, lane);
    } else if (lane == 0) {
        float* w = a.ws + (row * a.splits + sp) * (4 + 2 * a.top);
        w[0] = s.m; w[1] = s.l; w[2] = s.t;
        if (a.top == 0) w[3] = 0.0f;
    }
}

// Logical block = (row, split).  The split's elements are tiles of 1024 which its four wavefronts take in turn; a lane
// owns 16 of a tile, in runs of 4 (fp32) or 8 (bf16).
template <bool X32>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobArgs a, AtomArgs atom)
{
    constexpr int RUN = LogitRow<X32>::RUN, RUNS = 16 / RUN;
    __shared__ __attribute__((aligned(16))) uint64_t cand[LP_ROOM + LP_TOP + LP_PAD];
    __shared__ uint64_t chosen[LP_TOP];
    __shared__ Soft softs[4];
    __shared__ float nth[3][4];                   // per wavefront: its ceil(K / 4)-th, ceil(K / 2)-th and K-th largest lane maximum
    __shared__ uint4 tops[4][16];                 // the wavefronts' lane maxima, ordered
    __shared__ float peaks[LP_SEG][256];          // largest elements of the lanes' stretches
    __shared__ uint16_t sel[LP_SEG * 256];
    __shared__ int n_sel, n_cand;

    const uint32_t L = atom_logical_block(atom);
    const uint32_t S = a.splits;
    const int64_t row = S == 1 ? L : L / S;
    const uint32_t sp = S == 1 ? 0 : L % S;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles = (a.vocab + LP_TILE - 1) / LP_TILE;
    const int t0 = S == 1 ? 0 : (int)(sp * tiles / S), t1 = S == 1 ? tiles : (int)((sp + 1) * tiles / S);        // 64 * 2^20 at most
    const float c2 = a.scale * LOG2E;
    const int K = a.top;

    const LogitRow<X32> x_of{reinterpret_cast<const char*>(a.x) + row * a.ldx * (X32 ? 4 : 2), a.vocab};

    Soft s = {-INFINITY, 0.0f, 0.0f};            // m: a value near the largest one, see below
    float most = -INFINITY, peak = -INFINITY;     // the largest of this lane's elements, of its present stretch
    const int turns = (t1 - t0 + 3) / 4, len = max(1, (turns + LP_SEG - 1) / LP_SEG);
    int left = len, seg = 0;
    u32x4 raw[RUNS];
    if (t0 + wave < t1)
#pragma unroll
        for (int q = 0; q < RUNS; ++q) raw[q] = x_of.load(t0 + wave, lane, q);
    const int token = wave == 0 && S == 1 ? given_token(a, row) : -1;
    const float logit = token >= 0 ? logit_at<X32>(a, row, token) : 0.0f;
    for (int tile = t0 + wave; tile < t1; tile += 4) {
        float x[16];
#pragma unroll
        for (int q = 0; q < RUNS; ++q) x_of.unpack(raw[q], x + RUN * q);
        if (tile + 4 < t1)
#pragma unroll
            for (int q = 0; q < RUNS; ++q) raw[q] = x_of.load(tile + 4, lane, q);

        float mt = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, x[e]);
        peak = fmaxf(peak, mt);
        if (--left == 0 || tile + 4 >= t1) {                    // the stretch ends
            if (K) peaks[seg][tid] = peak;
            most = fmaxf(most, peak);
            peak = -INFINITY;
            left = len;
            ++seg;
        }
        // the sums' reference follows the largest value once that is 2^8 times as likely
        if (__any(s.m == -INFINITY ? mt > s.m : (mt - s.m) * c2 > 8.0f)) {
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
    }

    if (K) {
        const uint32_t mine = ordered(most);
        reinterpret_cast<uint32_t*>(tops[wave])[lane] = mine;
        wave_lds_sync();
        int above = 0;                            // (through scalar registers, a lane at a time, this took 4000 cycles)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint4 o = tops[wave][q];
            above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            // of the maxima that fewer than j lanes exceed the least one: with equal ones it is exceeded by fewer than j - 1
            int c = (K + (4 >> i) - 1) / (4 >> i) - 1;
            uint64_t at;
            while ((at = __ballot(above == c)) == 0) --c;
            if (lane == __ffsll((unsigned long long)at) - 1) nth[i][wave] = most;
        }
        if (tid == 0) n_sel = n_cand = 0;
    }
    s = soft_all<64>(s, c2);
    if (lane == 0) softs[wave] = s;
    __syncthreads();
    if (K) {
        const float lo01 = fminf(nth[1][0], nth[1][1]), hi01 = fmaxf(nth[1][0], nth[1][1]), lo23 = fminf(nth[1][2], nth[1][3]), hi23 = fmaxf(nth[1][2], nth[1][3]);
        float bound = fminf(fminf(nth[0][0], nth[0][1]), fminf(nth[0][2], nth[0][3]));
        bound = fmaxf(bound, fmaxf(fminf(hi01, hi23), fmaxf(lo01, lo23)));                 // second largest
        bound = fmaxf(bound, fmaxf(fmaxf(nth[2][0], nth[2][1]), fmaxf(nth[2][2], nth[2][3])));
        const float least = fmaxf(bound, -FLT_MAX);                                       // forbidden ones are no candidates
        // elements above `floor` (a key) of a run to the candidates
        auto offer = [&](const u32x4& v, int tile, int l, int q, uint64_t floor) {
            float x[RUN];
            uint32_t some = 0;
            x_of.unpack(v, x);
#pragma unroll
            for (int e = 0; e < RUN; ++e) some |= (x[e] >= least && top_key(x[e], x_of.index(tile, l, RUN * q + e)) > floor ? 1u : 0u) << e;
            if (some == 0) return;
            int at = atomicAdd(&n_cand, __popc(some));
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                if (some >> e & 1) {
                    if (at < LP_ROOM + LP_TOP) cand[at] = top_key(x[e], x_of.index(tile, l, RUN * q + e));
                    ++at;
                }
        };
        // of forbidden tokens, where fewer than K are allowed, the first K suffice
        auto fill = [&]() {
            const int i = t0 * LP_TILE + tid;
            if (bound == -INFINITY && tid < K && i < min(t1 * LP_TILE, a.vocab) && logit_at<X32>(a, row, i) == -INFINITY) cand[atomicAdd(&n_cand, 1)] = top_key(-INFINITY, i);
        };
        for (int g = 0; g < seg; ++g)
            if (peaks[g][tid] >= least) sel[atomicAdd(&n_sel, 1)] = (uint16_t)(g * 256 + tid);       // in any order: places follow from keys
        fill();
        __syncthreads();
        // item i, a run of a stretch
        auto scan = [&](int i, uint64_t floor) {
            const int who = sel[i / (RUNS * len)] & 255, g = sel[i / (RUNS * len)] >> 8, q = i % RUNS, tile = t0 + (who >> 6) + 4 * (g * len + i / RUNS % len);
            if (tile < t1) offer(x_of.load(tile, who & 63, q), tile, who & 63, q, floor);
        };
        const int items = n_sel * len * RUNS;
        for (int i = tid; i < items; i += 256) scan(i, 0);
        __syncthreads();
        int n = n_cand;
        if (n > LP_ROOM) {
            // many equal values: 256 items at a time, and only what is above the K-th chosen so far
            __syncthreads();
            if (tid == 0) n_cand = 0;
            __syncthreads();
            fill();
            n = 0;
            for (int i0 = 0; i0 < items; i0 += 256) {
                if (i0 + tid < items) scan(i0 + tid, n >= K ? chosen[K - 1] : 0);
                __syncthreads();
                n = n_cand;
                choose_top<256>(cand, n, K, chosen);
                __syncthreads();
                n = min(n, K);
                if (tid < n) cand[tid] = chosen[tid];
                if (tid == 0) n_cand = n;
                __syncthreads();
            }
        }
        choose_top<256>(cand, n, K, chosen);
        __syncthreads();
        n = min(n, K);
        save_top(a, row, sp, n, chosen);
    }
    if (wave != 0) return;
    s = soft_of_waves<4>(softs, lane, c2);
    save_sums(a, row, sp, s, token, logit, chosen, lane);
}

// The same where few workgroups meet a short piece (33 rows of 32003 bf16, top 32: 8.7 us): W wavefronts hold all of it, T tiles each, in registers.  All of it is
// on its way at once, the sums refer to the largest value itself, and nothing is read twice.  The candidates' bound is the
// `top`-th largest of the maxima of 64 to 127 groups of lanes.
template <bool X32, int W, int T>
__global__ __launch_bounds__(W * 64) void logprobs_held_kernel(LogprobArgs a, AtomArgs atom)
{
    constexpr int RUN = LogitRow<X32>::RUN, RUNS = 16 / RUN, NT = W * 64, TPG = NT / 128;         // threads to a group
    __shared__ __attribute__((aligned(16))) uint64_t cand[LP_ROOM + LP_TOP + LP_PAD];
    __shared__ uint64_t chosen[LP_TOP];
    __shared__ Soft softs[W];
    __shared__ __attribute__((aligned(16))) uint32_t peaks[128];      // largest elements of the groups, ordered
    __shared__ uint32_t bound_s;
    __shared__ int n_cand;

    const uint32_t L = atom_logical_block(atom), S = a.splits;
    const int64_t row = S == 1 ? L : L / S;
    const uint32_t sp = S == 1 ? 0 : L % S;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles = (a.vocab + LP_TILE - 1) / LP_TILE;
    const int t0 = S == 1 ? 0 : (int)(sp * tiles / S), t1 = S == 1 ? tiles : (int)((sp + 1) * tiles / S);        // at most W T tiles
    const float c2 = a.scale * LOG2E;
    const int K = a.top;
    const LogitRow<X32> x_of{reinterpret_cast<const char*>(a.x) + row * a.ldx * (X32 ? 4 : 2), a.vocab};

    u32x4 raw[T][RUNS];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int tile = t0 + wave + W * i;
        constexpr uint32_t none = X32 ? 0xff800000u : 0xff80ff80u;                  // -infinity
#pragma unroll
        for (int q = 0; q < RUNS; ++q) raw[i][q] = tile < t1 && x_of.whole(tile) ? x_of.load_whole(tile, lane, q) : u32x4{none, none, none, none};
    }
    if (t1 == tiles && !x_of.whole(tiles - 1) && (tiles - 1 - t0) % W == wave) {      // the row's end, which may break off anywhere
        u32x4 part[RUNS];
#pragma unroll
        for (int q = 0; q < RUNS; ++q) part[q] = x_of.load_partial(tiles - 1, lane, q);
#pragma unroll
        for (int i = 0; i < T; ++i)
            if (t0 + wave + W * i == tiles - 1)
#pragma unroll
                for (int q = 0; q < RUNS; ++q) raw[i][q] = part[q];
    }
    const int token = wave == 0 && S == 1 ? given_token(a, row) : -1;
    const float logit = token >= 0 ? logit_at<X32>(a, row, token) : 0.0f;
    if (tid == 0) { n_cand = 0; bound_s = ordered(-INFINITY); }

    const int busy = min(W, t1 - t0), group = busy >= 16 ? 16 : busy >= 8 ? 8 : busy >= 4 ? 4 : busy >= 2 ? 2 : 1;      // wavefronts with elements
    const int groups = busy * 64 / group;
    float most = -INFINITY, most_of[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        float x[16];
#pragma unroll
        for (int q = 0; q < RUNS; ++q) x_of.unpack(raw[i][q], x + RUN * q);
        most_of[i] = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most_of[i] = fmaxf(most_of[i], x[e]);
        most = fmaxf(most, most_of[i]);
    }
    Soft s = {0.0f, 0.0f, 0.0f};
    {
        const auto larger = [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); };
        uint32_t x = __float_as_uint(most), peak = x;
        x = lane_step<1>(x, larger); if (group >= 2) peak = x;
        x = lane_step<2>(x, larger); if (group >= 4) peak = x;
        x = lane_step<4>(x, larger); if (group >= 8) peak = x;
        x = lane_step<8>(x, larger); if (group >= 16) peak = x;
        x = lane_step<16>(x, larger);
        s.m = __uint_as_float(lane_step<32>(x, larger));
        if (K && wave < busy && lane % group == 0) peaks[tid / group] = ordered(__uint_as_float(peak));
        if (K && tid < 128 && tid >= groups) peaks[tid] = 0;                                 // less than any
    }
    const float ref = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
    for (int i = 0; i < T; ++i) {
        float x[16];
#pragma unroll
        for (int q = 0; q < RUNS; ++q) x_of.unpack(raw[i][q], x + RUN * q);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            // the difference first: products of masks of the type's lowest value overflow
            const float d = (x[e] - ref) * c2, p = __builtin_amdgcn_exp2f(d);
            s.l += p;
            s.t = fmaf(p, fmaxf(d, -300.0f), s.t);            // 0, not infinity times 0, for a forbidden token
        }
    }
    s.l = group_sum<64>(s.l);
    s.t = group_sum<64>(s.t);
    if (lane == 0) softs[wave] = s;
    __syncthreads();
    if (K) {
        {
            const uint32_t mine = peaks[tid / TPG];
            uint32_t above = 0, from = 0;
            for (int o = tid % TPG * 4; o < groups; o += TPG * 4) {
                const uint4 other = *reinterpret_cast<const uint4*>(peaks + o);
                above += (other.x > mine) + (other.y > mine) + (other.z > mine) + (other.w > mine);
                from += (other.x >= mine) + (other.y >= mine) + (other.z >= mine) + (other.w >= mine);
            }
            const auto add = [](uint32_t a, uint32_t b) { return a + b; };
            above = lane_group<TPG>(above, add);
            from = lane_group<TPG>(from, add);
            if (tid / TPG < groups && (int)above < K && (int)from >= K) bound_s = mine;      // the same of all who write
        }
        __syncthreads();
        const float bound = value_of(bound_s);
        const float least = fmaxf(bound, -FLT_MAX);                                       // forbidden ones are no candidates
        int total = 0;
#pragma unroll
        for (int i = 0; i < T; ++i)
            if (__any(most_of[i] >= least)) {
                float x[16];
#pragma unroll
                for (int q = 0; q < RUNS; ++q) x_of.unpack(raw[i][q], x + RUN * q);
#pragma unroll
                for (int e = 0; e < 16; ++e) total += __popcll(__ballot(x[e] >= least));
            }
        if (total) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&n_cand, total);    // in any order: places follow from keys
            at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
            for (int i = 0; i < T; ++i)
                if (__any(most_of[i] >= least)) {
                    float x[16];
#pragma unroll
                    for (int q = 0; q < RUNS; ++q) x_of.unpack(raw[i][q], x + RUN * q);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint64_t some = __ballot(x[e] >= least);
                        if (some == 0) continue;
                        const int mine = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0));
                        if (x[e] >= least && mine < LP_ROOM) cand[mine] = top_key(x[e], x_of.index(t0 + wave + W * i, lane, e));
                        at += __popcll(some);
                    }
                }
        }
        // of forbidden tokens, where fewer than K are allowed, the first K suffice
        auto fill = [&]() {
            const int i = t0 * LP_TILE + tid;
            if (bound == -INFINITY && tid < K && i < min(t1 * LP_TILE, a.vocab) && logit_at<X32>(a, row, i) == -INFINITY) {
                const int at = atomicAdd(&n_cand, 1);
                if (at < LP_ROOM) cand[at] = top_key(-INFINITY, i);
            }
        };
        fill();
        __syncthreads();
        int n = n_cand;
        if (n > LP_ROOM) {
            // many equal values: an element per thread at a time, and only what is above the K-th chosen so far
            __syncthreads();
            if (tid == 0) n_cand = 0;
            __syncthreads();
            fill();
            n = 0;
            for (int i0 = t0 * LP_TILE; i0 < min(t1 * LP_TILE, a.vocab); i0 += NT) {
                const int i = i0 + tid;
                const float x = i < min(t1 * LP_TILE, a.vocab) ? logit_at<X32>(a, row, i) : -INFINITY;
                if (x >= least) {
                    const uint64_t k = top_key(x, i);
                    if (k > (n >= K ? chosen[K - 1] : 0)) cand[atomicAdd(&n_cand, 1)] = k;      // NT and K at most
                }
                __syncthreads();
                n = n_cand;
                choose_top<NT>(cand, n, K, chosen);
                __syncthreads();
                n = min(n, K);
                if (tid < n) cand[tid] = chosen[tid];
                if (tid == 0) n_cand = n;
                __syncthreads();
            }
        }
        choose_top<NT>(cand, n, K, chosen);
        __syncthreads();
        save_top(a, row, sp, min(n, K), chosen);
    }
    if (wave != 0) return;
    s = soft_of_waves<W>(softs, lane, c2);
    save_sums(a, row, sp, s, token, logit, chosen, lane);
}

// Joins the splits of a row: one workgroup per row.  With j = ceil(top / splits) at least `top` keys reach the least of the
// largest j-th keys of ceil(top / j) groups of splits; the few that do find their places by counting larger ones.
template <bool X32>
__global__ __launch_bounds__(256) void logprobs_merge_kernel(LogprobArgs a, AtomArgs atom)
{
    __shared__ __attribute__((aligned(16))) uint64_t cand[LITHOS_LOGPROBS_MAX_SPLITS * LP_TOP + LP_PAD];
    __shared__ uint64_t chosen[LP_TOP], bound_s;
    __shared__ int n_cand;
    const int64_t row = atom_logical_block(atom);
    const int tid = threadIdx.x, lane = tid & 63;
    const float c2 = a.scale * LOG2E;
    const int K = a.top, S = a.splits, stride = 4 + 2 * K;
    const float* const ws = a.ws + row * S * stride;
    auto key_at = [&](int sp, int j) {
        const uint2 k = reinterpret_cast<const uint2*>(ws + sp * stride + 4)[j];
        return ((uint64_t)k.y << 32) | k.x;
    };
    // everything is fetched at once: the splits' sums and j-th keys, this thread's first key, the given token's logit
    Soft s = {-INFINITY, 0.0f, 0.0f};
    const int t = given_token(a, row);
    float logit = 0.0f;
    uint64_t mine = 0;
    if (tid < S * K) mine = key_at(tid / K, tid % K);
    const int mine_of = tid < S * K ? (int)ws[tid / K * stride + 3] : 0;
    const int j = K ? (K + S - 1) / S : 1, m = K ? (K + j - 1) / j : 1;
    if (tid < 64) {
        const f32x4_b4 p = lane < S ? *reinterpret_cast<const f32x4_b4*>(ws + lane * stride) : f32x4_b4{-INFINITY, 0.0f, 0.0f, 0.0f};
        uint64_t jth = K && lane < S ? key_at(lane, j - 1) : 0;
        if (t >= 0) logit = logit_at<X32>(a, row, t);
        if (K) {
            if ((int)p.w < j) jth = 0;
            const uint32_t v = least_of_groups((uint32_t)(jth >> 32), power_of_two_from(m));         // 0: not as many splits
            if (lane == 0) { n_cand = 0; bound_s = (uint64_t)v << 32; }
        }
        s = soft_all<64>(Soft{p.x, p.y, p.z}, c2);
    }
    if (K) {
        __syncthreads();
        const uint64_t bound = bound_s;
        for (int i = tid; i < S * K; i += 256) {
            const int sp = i / K, q = i % K;
            const bool there = q < (i == tid ? mine_of : (int)ws[sp * stride + 3]);
            const uint64_t k = !there ? 0 : i == tid ? mine : key_at(sp, q);
            if (there && k >= bound) cand[atomicAdd(&n_cand, 1)] = k;           // in any order: places follow from the keys
        }
        __syncthreads();
        const int n = n_cand;
        choose_top<256>(cand, n, K, chosen);
        if (tid >= n && tid < K) chosen[tid] = top_key(-INFINITY, tid);         // rows with NaN: any token
        __syncthreads();
    }
    if (tid < 64) write_row(a, row, s, logit, t >= 0, chosen, lane);
}

// ---- gradient ------------------------------------------------------------------------
//   dx_i = c (g_lp (1[i = t] - p_i) - g_H p_i (log p_i + H)),   log p_i = c x_i - lse
// with lse and H from the forward pass.  A forbidden token (x = -inf) and a row without allowed ones get 0.  Bound by the bytes
// read and written: 1024 rows of 50001 fp32 take 78 us, 5.3 TB/s.
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
        // p is 0 well above -300; a mask of the type's lowest value must not become 0 times infinity below
        const float lp = fmaxf(fmaf(c, x[e], -lse), -300.0f), p = __builtin_amdgcn_exp2f(lp * LOG2E);
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

// Wavefronts and tiles of each that hold a workgroup's piece, 0: it is read as a stream.  Held by 16 wavefronts where each has a
// CU for itself (33 rows of 32003, top 32, 11.8 -> 8.7 us a pass; 1 of 16384 7.5 -> 6.0; 200 of 50001 13.7 -> 12.6; more rows
// are as fast as a stream: 300 of 50001 20.8 whole).  Eight tiles spill: 200 rows of 131072 took 59 us, as a stream 22.
struct Held { int waves, tiles; };
static Held lp_held(const lithos_op_t& op)
{
    const int64_t splits = std::max<int64_t>(1, op.dim[3]), blocks = op.dim[0] * splits;
    const int64_t piece = ((op.dim[1] + LP_TILE - 1) / LP_TILE + splits - 1) / splits;         // tiles
    if (op.kind != LITHOS_OP_LOGPROBS) return {0, 0};
    if (piece <= 4) return {4, 1};
    if (blocks > 256 || piece > 64) return {0, 0};
    return {16, piece <= 16 ? 1 : piece <= 32 ? 2 : 4};
}

template <bool X32>
static lp_fn lp_pick(const lithos_op_t& op)
{
    const Held h = lp_held(op);
    if (h.waves == 4) return logprobs_held_kernel<X32, 4, 1>;
    return h.tiles == 1 ? logprobs_held_kernel<X32, 16, 1> : h.tiles == 2 ? logprobs_held_kernel<X32, 16, 2> : h.tiles == 4 ? logprobs_held_kernel<X32, 16, 4> : logprobs_kernel<X32>;
}

static lp_fn lp_kernel(const lithos_op_t& op)
{
    const bool x32 = op.flags & LITHOS_F_IN_F32;
    if (op.kind == LITHOS_OP_LOGPROBS) return x32 ? lp_pick<true>(op) : lp_pick<false>(op);
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
    if (op.flags & ~(LITHOS_F_IN_F32 | (grad ? LITHOS_F_OUT_F32 : 0u)))
        return fail(LITHOS_EINVAL, grad ? "logprobs_grad: takes IN_F32 and OUT_F32 only" : "logprobs: takes IN_F32 only");
    // exponents are of two: a scale whose product with log2(e) is infinite would make NaN of equal logits
    if (!(op.fparam[0] > 0.0f) || !(op.fparam[0] * LOG2E < INFINITY)) return fail(LITHOS_EINVAL, "logprobs: the scale (fparam0) must be positive and below 2.3e38");
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
        blocks = merge ? (uint64_t)rows : (uint64_t)rows * splits;
    }
    if (blocks > 0x7fffffffull) return fail(LITHOS_EINVAL, "logprobs: too many workgroups");
    plan->grid = {(uint32_t)blocks, 1, 1};
    plan->total = (uint32_t)blocks;
    if (!grad && lp_held(op).waves) plan->threads = 64 * lp_held(op).waves;
    plan->wg_per_cu = cached_occupancy(grad ? (const void*)lp_grad_kernel(op) : (const void*)lp_kernel(op), (int)plan->threads, 4);
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

// Rows of up to 65536 tokens stay whole: a second launch costs more than it saves (us a pass, whole / best split: 33 x 32003
// 8.7 / 11.2, 64 x 50257 11.2 / 11.1, 250 x 65536 15.8 / 20, 400 x 50001 17 / 20).  Longer ones are cut into a piece for each
// CU, at least two, of a tile of 1024 for each of four wavefronts: 4 x 131072 21 / 9.7 (32 pieces), 64 x 131072 22 / 12.5 (4),
// 128 x 131072 22 / 16.4 (2), 300 x 131072 27.4 / 26.2 (2); 400 x 131072 31 / 32.
int logprobs_split_hint(const lithos_op_t& op, int n_cus)
{
    const int64_t rows = op.dim[0], quads = (op.dim[1] + 4 * LP_TILE - 1) / (4 * LP_TILE);
    if (op.dim[1] <= 64 * LP_TILE || 2 * rows >= 3ll * n_cus) return 1;
    return (int)std::min({quads, std::max<int64_t>(2, (n_cus + rows - 1) / rows), (int64_t)LITHOS_LOGPROBS_MAX_SPLITS});
}

} // namespace lithos
