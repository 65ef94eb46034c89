// beam_select: the best continuations of an item's beams, from their logits.
//
// s(b, t) = c_b + x_bt - lse_b, lse_b = log sum_t exp(x_bt).  Within a beam the order is that of the logits, which are exact; between
// beams it hangs on the lse, sums in fp32 whose error is known (near_of): where two beams' scores are nearer than that, the sums
// in question are made again in 64 bits.  So which tokens are picked does not hang on rounding.  Scores are c_b + ((x_bt - max) - log of
// the sum against it): beams whose logits differ by a constant tie, as they should.
//
// Two kernels.  beam_scan_kernel reads the logits once: a workgroup to a piece of a row, held in registers, gives the piece's maximum,
// its sum of exponentials, and its n_out largest logits.  beam_pick_kernel, a workgroup to an item, joins the sums and picks from the
// pieces' largest.
#include "beams.h"

#include <float.h>

#include <cmath>

#include "kv.h"
#include "wave.h"

namespace llmint8 {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float NONE = -__builtin_inff();

struct Pick {  // a logit and its token
    float x;
    int t;
};

// Floats as unsigned integers in the same order.
__device__ __forceinline__ unsigned order_key(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// The value of a key whose last bits are cleared; -inf where that is none: -inf's key without its last bits, and any below, would be a NaN,
// which nothing is above.
__device__ __forceinline__ float bound_of(unsigned k)
{
    return k < order_key(-FLT_MAX) ? NONE : __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A value that is not above the k-th largest of the wave's 64, and not far below: the key's last LOW bits are left open.  (Two bits at a time,
// three counts that do not wait for each other: more code and 0.5 us slower in both kernels.)
template <int LOW>
__device__ __forceinline__ float not_above_kth(float x, int k)
{
    const unsigned key = order_key(x);
    unsigned at = 0;
#pragma unroll
    for (int bit = 31; bit >= LOW; bit--) {
        const unsigned c = at | (1u << bit);
        if (__popcll(__ballot(key >= c)) >= k) at = c;
    }
    return bound_of(at);
}

__device__ __forceinline__ float wave_max(float x)
{
    return wave_reduce(x, NONE, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ double wave_sum(double x)
{
    return wave_reduce(x, 0.0, [](double a, double b) { return a + b; });
}

// The k <= 64 best of what a wave is shown, best first, one to a lane: larger values, of equal ones the lower place.
template <class V, class I>
struct Best {
    V v;
    I at;
    int k;
    V last;  // the k-th
    I last_at;

    __device__ __forceinline__ explicit Best(int n) : v(-__builtin_inf()), at(-1), k(n), last(-__builtin_inf()), last_at(-1) {}
    __device__ __forceinline__ bool takes(V x, I i) const { return x > last || (x == last && i < last_at); }
    __device__ __forceinline__ void add(V x, I i)  // the same in all lanes, and takes(x, i)
    {
        const int lane = threadIdx.x & 63;
        const int pos = __popcll(__ballot(lane < k && (v > x || (v == x && at < i))));
        const V pv = __shfl_up(v, 1);
        const I pa = __shfl_up(at, 1);
        v = lane == pos ? x : lane > pos ? pv : v;
        at = lane == pos ? i : lane > pos ? pa : at;
        last = __shfl(v, k - 1);
        last_at = __shfl(at, k - 1);
    }
};

typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f8v __attribute__((ext_vector_type(8)));
template <class T>
struct Of;
template <>
struct Of<_Float16> {
    typedef h8v v8;
    static constexpr float LOWEST = -65504.0f;
    static __device__ __forceinline__ v8 load(const _Float16* p) { return __builtin_bit_cast(h8v, load8((const unsigned short*)p)); }
    static __device__ __forceinline__ float largest(v8 v)
    {
        const u4 w = __builtin_bit_cast(u4, v);
        const h2 m = __builtin_bit_cast(h2, pk_max_f16(pk_max_f16(w[0], w[1]), pk_max_f16(w[2], w[3])));
        return __builtin_fmaxf((float)m[0], (float)m[1]);
    }
    // v without its first d elements
    static __device__ __forceinline__ v8 without(v8 v, int d)
    {
        u4 w = __builtin_bit_cast(u4, v);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const unsigned upper = (w[q] & 0xffff0000u) | 0xfc00u;
            w[q] = d >= 2 * q + 2 ? 0xfc00fc00u : d == 2 * q + 1 ? upper : w[q];
        }
        return __builtin_bit_cast(v8, w);
    }
    // sum of exp(x - M), M >= every x: 2^(x log2 e - r) with r = M log2 e rounded, which beyond() makes good.  A conversion, a product and a
    // difference in one instruction, with one rounding.
    struct Exp {
        float r;
        __device__ __forceinline__ explicit Exp(float M) : r(M * LOG2E) {}
        __device__ __forceinline__ float of(v8 v) const
        {
            const u4 w = __builtin_bit_cast(u4, v);
            float t[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel_hi:[1,0,0]" : "=v"(t[2 * e]) : "v"(w[e]), "s"(LOG2E), "v"(r));
                asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(t[2 * e + 1]) : "v"(w[e]), "s"(LOG2E), "v"(r));
            }
#pragma unroll
            for (int e = 0; e < 8; e++) t[e] = __builtin_amdgcn_exp2f(t[e]);
            return ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
        // ln of what a sum against M is too large by
        static __device__ __forceinline__ double beyond(float M) { return ((double)M * LOG2E - (double)(M * LOG2E)) * 0.69314718055994530942; }
    };
};
template <>
struct Of<float> {
    typedef f8v v8;
    static constexpr float LOWEST = -FLT_MAX;
    typedef f8v at4 __attribute__((aligned(4)));
    static __device__ __forceinline__ v8 load(const float* p) { return *(const at4*)p; }
    static __device__ __forceinline__ float largest(v8 v)
    {
        float m = v[0];
#pragma unroll
        for (int e = 1; e < 8; e++) m = __builtin_fmaxf(m, v[e]);
        return m;
    }
    static __device__ __forceinline__ v8 without(v8 v, int d)
    {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = e < d ? NONE : v[e];
        return v;
    }
    struct Exp {  // (products could be beyond fp32's range: the difference first)
        float M;
        __device__ __forceinline__ explicit Exp(float m) : M(m) {}
        __device__ __forceinline__ float of(v8 v) const
        {
            float t[8];
#pragma unroll
            for (int e = 0; e < 8; e++) t[e] = __builtin_amdgcn_exp2f((v[e] - M) * LOG2E);
            return ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
        static __device__ __forceinline__ double beyond(float) { return 0.0; }
    };
};

// A row's beam has logits to look at.  (NaN and +inf as a score: beam_pick_kernel tells of it.)
__device__ __forceinline__ bool lives(const BeamArgs& a, long long row)
{
    const float c = a.scores[row];
    return c > NONE && c <= FLT_MAX && !(a.ended && a.ended[row]);
}

// exp(x) for x <= 0, within some units of 1e-16: x = n ln 2 + r, |r| <= ln 2 / 2, the series to r^12 (the rest is below 2e-16).  ln 2 in two
// parts, as Cody and Waite reduce arguments (Software Manual for the Elementary Functions, 1980): floor(2^32 ln 2) / 2^32, which n times is
// exact, and what is left.
__device__ __forceinline__ double exp_of(double x)
{
    x = __builtin_fmax(x, -1000.0);
    const double n = __builtin_rint(x * 1.4426950408889634074);
    double r = __builtin_fma(n, -2977044471.0 / 4294967296.0, x);
    r = __builtin_fma(n, -0x1.a39ef35793c76p-33, r);
    constexpr double c[12] = {1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
    double p = 1.0 / 479001600.0;
#pragma unroll
    for (int i = 0; i < 12; i++) p = __builtin_fma(p, r, c[i]);
    return __builtin_ldexp(p, (int)n);
}

struct Sum {
    double s;  // of the piece's exponentials against max
    float max;
};

// Picks as integers in their order: larger logits, of equal ones the lower token (-0 and 0 are equal).
__device__ __forceinline__ unsigned long long pick_key(const Pick& p)
{
    return (unsigned long long)order_key(p.x + 0.0f) << 32 | (unsigned)~p.t;
}

constexpr int SHOWN = 96;  // groups of 8 logits that a wave's largest are picked from
constexpr int FEW = 128;   // those of their logits that are not below the bound: little more than what is kept, mostly

// G groups of 8 logits to a thread: a wave's lanes side by side, the waves side by side, then the groups, so that a piece is
// read in runs of 4 KiB (fp16).  The waves work by themselves until their largest are joined at the end, behind the only barrier.
// Bound by HBM and by vector instructions, about equally: 512 rows of 131072 fp16 logits, 134 MB, in 27 to 28 us, 4.9 TB/s (a read: 6.6); a
// wave's 4 096 logits are 64 exponentials of four turns and some 500 other instructions.  Where rows are few, by latency: the parts
// of a workgroup's 5 to 8 us are the logits (1 to 2), maximum and bound (1), exponentials (0.8), the join (1).
template <class T, int G>
__global__ void __launch_bounds__(THREADS) beam_scan_kernel(const BeamArgs a, const Div parts, int keep, Sum* __restrict__ sums, Pick* __restrict__ picks)
{
    typedef Of<T> O;
    typedef typename O::v8 v8;
    __shared__ float s_max[WAVES];
    __shared__ double s_sum[WAVES];
    __shared__ int s_n[WAVES];
    __shared__ v8 s_shown[WAVES][SHOWN];
    __shared__ int s_shown_at[WAVES][SHOWN];
    __shared__ Pick s_few[WAVES][FEW], s_best[WAVES * LLMINT8_BEAM_MAX];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = parts.quot((int)blockIdx.x), part = (int)blockIdx.x - row * (int)parts.d;
    if (!lives(a, row)) return;
    const T* const src = (const T*)a.logits + row * a.ld;
    const int vocab = a.vocab, start = part * (8 * THREADS * G);
    const unsigned long long below = (1ull << lane) - 1;

    // First token of group g of a lane.  The row's last piece: a group that reaches past the row's end is its last 8 tokens instead,
    // without those that come before the group.
    const bool last = vocab - start < 8 * THREADS * G;
    auto meant = [&](int g, int l) { return start + g * (8 * THREADS) + 512 * w + 8 * l; };
    auto first = [&](int g, int l) {
        const int t = meant(g, l), most = vocab - 8;
        return t < most ? t : most < 0 ? 0 : most;
    };
    v8 x[G];
    if (vocab >= 8) {
#pragma unroll
        for (int g = 0; g < G; g++) x[g] = O::load(src + first(g, lane));
        if (last)
#pragma unroll
            for (int g = 0; g < G; g++) x[g] = O::without(x[g], meant(g, lane) - first(g, lane));
    } else {
#pragma unroll
        for (int g = 0; g < G; g++)
#pragma unroll
            for (int e = 0; e < 8; e++) x[g][e] = g == 0 && tid == 0 && e < vocab ? src[e < vocab ? e : 0] : (T)NONE;
    }

    float top[G], m = NONE;
#pragma unroll
    for (int g = 0; g < G; g++) {
        top[g] = O::largest(x[g]);
        m = __builtin_fmaxf(m, top[g]);
    }
    // `keep` lanes have a logit that is not below tau: nothing below it is wanted.  The groups that have others go to LDS.
    const float tau = __builtin_fmaxf(not_above_kth<16>(m, keep), -FLT_MAX);
    v8* const shown = s_shown[w];
    int* const shown_at = s_shown_at[w];
    int groups = 0;
#pragma unroll
    for (int g = 0; g < G; g++) {
        const unsigned long long hits = __ballot(top[g] >= tau);
        const int slot = groups + __popcll(hits & below);
        if (top[g] >= tau && slot < SHOWN) shown[slot] = x[g], shown_at[slot] = first(g, lane);
        groups += __popcll(hits);
    }

    // (A mask of the type's lowest value is a logit like others: the reference is the maximum itself, -inf apart.)
    const float M = __builtin_fmaxf(wave_max(m), O::LOWEST);
    const typename O::Exp ex(M);
    double sum = 0.0;
#pragma unroll
    for (int g = 0; g < G; g++) sum += (double)ex.of(x[g]);
    sum = wave_sum(sum);
    if (lane == 0) s_max[w] = M, s_sum[w] = sum;

    wave_order();
    Pick* const few = s_few[w];
    Pick* const best = s_best + w * keep;
    int n = 0;
    if (groups <= SHOWN)
        for (int t0 = 0; t0 < 8 * groups; t0 += 64) {
            const int t = t0 + lane;
            const float v = t < 8 * groups ? (float)((const T*)shown)[t] : NONE;
            const unsigned long long hits = __ballot(v >= tau);
            const int at = n + __popcll(hits & below);
            if (v >= tau && at < FEW) few[at] = {v, shown_at[t >> 3] + (t & 7)};
            n += __popcll(hits);
        }
    if (groups <= SHOWN && n <= FEW) {
        wave_order();
        unsigned long long key[FEW / 64];
        Pick mine[FEW / 64];
        int rank[FEW / 64] = {};
#pragma unroll
        for (int k = 0; k < FEW / 64; k++) {
            mine[k] = few[64 * k + lane < n ? 64 * k + lane : 0];
            key[k] = 64 * k + lane < n ? pick_key(mine[k]) : 0;
        }
#pragma unroll
        for (int k = 0; k < FEW / 64; k++)
            for (int q = 0; q < n - 64 * k && q < 64; q += 4) {  // (keys of 0 behind the last count for nothing)
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    const unsigned long long o = lane_of(key[k], q + u);
#pragma unroll
                    for (int y = 0; y < FEW / 64; y++) rank[y] += o > key[y];
                }
            }
#pragma unroll
        for (int k = 0; k < FEW / 64; k++)
            if (64 * k + lane < n && rank[k] < keep) best[rank[k]] = mine[k];
        n = n < keep ? n : keep;
    } else {
        // Many equal logits, or large ones far apart: group by group, best first, so that a group has at most `keep` to add.
        Best<float, int> found(keep);
#pragma unroll 1
        for (int g = 0; g < G; g++) {
            v8 y = x[0];
#pragma unroll
            for (int q = 1; q < G; q++)
                if (q == g) y = x[q];
            unsigned left = 0xff;
            for (;;) {
                float v = NONE;
                int e = 0;
#pragma unroll
                for (int q = 7; q >= 0; q--)
                    if ((left >> q & 1) && (float)y[q] >= v) v = (float)y[q], e = q;
                const float V = wave_max(v);
                if (!(V > found.last)) break;
                const int l = __ffsll(__ballot(v == V)) - 1;
                if (lane == l) left &= ~(1u << e);
                found.add(V, first(g, l) + __shfl(e, l));
            }
        }
        if (lane < keep) best[lane] = {found.v, found.at};
        n = __popcll(__ballot(lane < keep && found.v > NONE));
    }
    if (lane == 0) s_n[w] = n;
    __syncthreads();

    const long long at = (long long)row * parts.d + part;
    const int all = WAVES * keep;
    auto listed = [&](int i) { return i < all && i % keep < s_n[i < all ? i / keep : 0]; };
    if (64 * w < all) {
        const bool there = listed(tid);
        const Pick mine = s_best[there ? tid : 0];
        const unsigned long long own = pick_key(mine);
        int rank = 0;
        for (int q0 = 0; q0 < all; q0 += 64) {
            const unsigned long long key = listed(q0 + lane) ? pick_key(s_best[q0 + lane]) : 0;
            for (int q = 0; q < all - q0 && q < 64; q += 4) {
#pragma unroll
                for (int u = 0; u < 4; u++) rank += lane_of(key, q + u) > own;
            }
        }
        if (there && rank < keep) picks[at * keep + rank] = mine;
    }
    const int total = s_n[0] + s_n[1] + s_n[2] + s_n[3];
    if (tid >= total && tid < keep) picks[at * keep + tid] = {NONE, -1};
    if (w == WAVES - 1) {
        const float max4 = __builtin_fmaxf(__builtin_fmaxf(s_max[0], s_max[1]), __builtin_fmaxf(s_max[2], s_max[3])), own = s_max[lane & 3];
        const double part_sum = lane < WAVES ? s_sum[lane] * exp_of(((double)own - (double)max4) - O::Exp::beyond(own)) : 0.0;
        const double s = wave_sum(part_sum);
        if (lane == 0) sums[at] = {s, max4};
    }
}

constexpr int PICK_THREADS = 512, PICK_WAVES = PICK_THREADS / 64;
constexpr int SOME = PICK_THREADS;  // candidates that are ranked by counting: one a thread

// A score and its place among equal ones: the beam, then larger logits (64 bits of a score need not tell fp32 logits apart), then the
// token.
struct Candidate {
    double s;
    unsigned long long at;

    static constexpr int TOKEN_BITS = 27;
    static_assert(LLMINT8_BEAM_MAX <= 32 && LLMINT8_BEAM_MAX_VOCAB <= 1 << TOKEN_BITS, "5 bits of beam, 32 of logit, 27 of token");
    __device__ __forceinline__ void place(int b, float x, int t)
    {
        at = (unsigned long long)b << (32 + TOKEN_BITS) | (unsigned long long)~order_key(x + 0.0f) << TOKEN_BITS | (unsigned)t;
    }
    __device__ __forceinline__ int beam() const { return (int)(at >> (32 + TOKEN_BITS)); }
    __device__ __forceinline__ int token() const { return (int)at & ((1 << TOKEN_BITS) - 1); }
};

// A workgroup to an item: latency, 5 to 8 us of dependent steps (2.4 of them the launch): sums of the rows, scores and a bound, the
// candidates above it, their ranks.  near: two scores of different beams that are not further apart are compared by sums in 64 bits
// (near_of), which takes 20 us for each row of 131072.  That is rare: fp16 logits are a grid, and where two beams' sums differ by about a
// multiple of its step, candidates of both can be near each other (1 of 192 items with 32 picked of 8 beams).
template <class T>
__global__ void __launch_bounds__(PICK_THREADS) beam_pick_kernel(const BeamArgs a, const Div parts, const Div per_row, double near,
                                                                 const Sum* __restrict__ sums, const Pick* __restrict__ picks)
{
    constexpr int B = LLMINT8_BEAM_MAX;
    enum { DEAD, LIVE, ENDED };
    __shared__ double s_log[B], s_cum[B], s_part[PICK_WAVES];  // s_log: of the sum of exp(x - maximum)
    __shared__ float s_max[B], s_tau[PICK_WAVES], s_share[PICK_WAVES];
    __shared__ int s_state[B], s_n;
    __shared__ unsigned s_redo;  // a bit for each beam: its sum is to be made again
    __shared__ Candidate some[SOME], top[B];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long row0 = (long long)blockIdx.x * a.beams;
    const double none = -__builtin_inf();
    const int C = a.beams * (int)per_row.d;  // the pieces' largest; behind them one candidate for each beam that has ended

    const Pick held = picks[row0 * per_row.d + (tid < C ? tid : C - 1)];  // (requested before what it hangs on; a row without any has whatever
                                                                          // the workspace had)

    // sums of the rows
    for (int b = w; b < a.beams; b += PICK_WAVES) {
        const long long row = row0 + b;
        const Sum first = sums[row * parts.d + (lane < (int)parts.d ? lane : 0)];
        const float c = a.scores[row];
        int state = a.ended && a.ended[row] ? ENDED : LIVE;
        bool bad = !(c <= FLT_MAX);  // NaN, +inf
        if (bad || c == NONE) state = DEAD;
        float M = NONE;
        double log_sum = 0.0;
        if (state == LIVE) {
            M = lane < (int)parts.d ? first.max : NONE;
            for (int q = lane + 64; q < (int)parts.d; q += 64) M = __builtin_fmaxf(M, sums[row * parts.d + q].max);
            M = wave_max(M);
            auto one = [&](const Sum& v) { return v.s * exp_of((double)v.max - (double)M); };
            double s = lane < (int)parts.d ? one(first) : 0.0;
            for (int q = lane + 64; q < (int)parts.d; q += 64) s += one(sums[row * parts.d + q]);
            s = wave_sum(s);
            // NaN, or +inf (whose distance to itself is NaN), anywhere in the row makes the sum NaN.  Nothing but masked tokens: 0
            if (!(s <= DBL_MAX)) bad = true;
            if (bad || s == 0.0) state = DEAD;
            log_sum = log(s);
        }
        if (lane == 0) {
            s_log[b] = log_sum, s_cum[b] = c, s_max[b] = M, s_state[b] = state;
            if (bad && a.status) atomicOr(a.status, LLMINT8_BEAM_NOT_FINITE);
        }
    }
    __syncthreads();

    auto candidate = [&](int c, Pick p) {
        Candidate r = {none, 0};
        if (c < C) {
            const int b = per_row.quot(c);
            if (s_state[b] == LIVE && p.t >= 0) {
                r.place(b, p.x, p.t);
                r.s = s_cum[b] + (((double)p.x - (double)s_max[b]) - s_log[b]);
            }
        } else if (s_state[c - C] == ENDED) {
            r.place(c - C, 0.0f, a.eos);
            r.s = s_cum[c - C];
        }
        return r;
    };
    auto pick_of = [&](int c) { return picks[row0 * per_row.d + (c < C ? c : C - 1)]; };
    const int all = C + a.beams;
    Candidate mine;
    auto each = [&](auto f) {  // (one of a thread's candidates is kept in registers: the code of four took 0.5 us longer)
        if (tid < all) f(mine);
        for (int c = tid + PICK_THREADS; c < all; c += PICK_THREADS) f(candidate(c, pick_of(c)));
    };

    unsigned exact = 0;
    for (int b = 0; b < a.beams; b++) exact |= s_state[b] == LIVE ? 0u : 1u << b;
    const unsigned every = a.beams < 32 ? (1u << a.beams) - 1 : ~0u;
    int found;
    for (;;) {
        if (tid == 0) s_n = 0, s_redo = 0;
        if (tid < all) mine = candidate(tid, held);
        double m = none;
        each([&](const Candidate& r) { m = __builtin_fmax(m, r.s); });
        // Two bounds below the n_out-th: the largest of the waves' own, and, where many are picked, the smallest of those that each of the
        // waves that all have candidates has its share above.
        const float best_of_thread = __double2float_rd(m), tau_w = not_above_kth<14>(best_of_thread, a.n_out);
        const int full = all / 64 < PICK_WAVES ? all / 64 : PICK_WAVES;
        const bool shares = a.n_out > 8 && full > 1;
        const float share_w = shares && w < full ? not_above_kth<14>(best_of_thread, (a.n_out + full - 1) / full) : -NONE;
        if (lane == 0) s_tau[w] = tau_w, s_share[w] = share_w;
        __syncthreads();
        float t = s_tau[0], share = s_share[0];
#pragma unroll
        for (int q = 1; q < PICK_WAVES; q++) t = __builtin_fmaxf(t, s_tau[q]), share = __builtin_fminf(share, s_share[q]);
        if (shares) t = __builtin_fmaxf(t, share);
        const double tau = (double)t - 1.01 * near;  // what is picked, and what it may have to be told from
        each([&](const Candidate& r) {
            if (r.s >= tau && r.s > none) {
                const int at = atomicAdd(&s_n, 1);
                if (at < SOME) some[at] = r;
            }
        });
        __syncthreads();
        int n = s_n;
        const bool many = n > SOME, all_exact = exact == every;
        if (many && all_exact) {
            Best<double, unsigned long long> best(a.n_out);
            for (int c0 = 64 * w; c0 < all; c0 += PICK_THREADS) {
                Candidate r = {none, 0};
                if (c0 + lane < all) r = candidate(c0 + lane, pick_of(c0 + lane));
                for (;;) {
                    const unsigned long long take = __ballot(r.s > none && best.takes(r.s, r.at));
                    if (!take) break;
                    const int l = __ffsll(take) - 1;
                    best.add(__shfl(r.s, l), __shfl(r.at, l));
                    if (lane == l) r.s = none;
                }
            }
            if (lane < a.n_out) some[w * a.n_out + lane] = {best.v, best.at};
            n = PICK_WAVES * a.n_out;
            __syncthreads();
        }
        if (!many && n > 128) {
            // Ranking takes time by their number: the bound again, over all of them, first.
            const Candidate one = some[tid < n ? tid : 0];
            const unsigned key = tid < n ? order_key(__double2float_rd(one.s)) : 0u;
            unsigned at = 0;
            for (int bit = 31; bit >= 14; bit--)
                if (__syncthreads_count(key >= (at | 1u << bit)) >= a.n_out) at |= 1u << bit;
            if (tid == 0) s_n = 0;
            __syncthreads();
            // (scores below fp32's range are -inf here and are all kept)
            if (tid < n && one.s >= (double)bound_of(at) - 1.01 * near) some[atomicAdd(&s_n, 1)] = one;
            __syncthreads();
            n = s_n;
        }
        found = 0;
        if (!many || all_exact) {
            const Candidate one = some[tid < n ? tid : 0];
            const bool counts = tid < n && one.s > none;
            if (64 * w < n) {
                int rank = 0;
                unsigned close = 0;  // beams that have a candidate near this one
                const unsigned long long own = one.at;
                const int beam = one.beam();
                for (int q0 = 0; q0 < n; q0 += 64) {
                    const Candidate o = some[q0 + lane < n ? q0 + lane : 0];
                    const double s = q0 + lane < n ? o.s : none;
                    const int end = n - q0 < 64 ? n - q0 : 64;
                    for (int q = 0; q < end; q += 4) {  // (none behind the last)
#pragma unroll
                        for (int u = 0; u < 4; u++) {
                            const Candidate other = {lane_of(s, q + u), lane_of(o.at, q + u)};
                            rank += other.s > one.s || (other.s == one.s && other.at < own);
                            close |= __builtin_fabs(other.s - one.s) <= near ? 1u << other.beam() : 0u;
                        }
                    }
                }
                if (counts && rank < a.n_out) {
                    top[rank] = one;
                    close &= ~(1u << beam);
                    const unsigned redo = (close & ~exact) | (close && !(exact >> beam & 1) ? 1u << beam : 0u);
                    if (redo) atomicOr(&s_redo, redo);
                }
            }
            found = __syncthreads_count(counts);
            found = found < a.n_out ? found : a.n_out;
        } else {  // too many to compare them
            if (tid == 0) s_redo = every & ~exact;
            __syncthreads();
        }
        const unsigned redo = s_redo;
        if (!redo) break;
        for (int b = 0; b < a.beams; b++) {
            if (!(redo >> b & 1)) continue;
            const T* const src = (const T*)a.logits + (row0 + b) * a.ld;
            const double M = s_max[b];
            double s = 0.0;
            int t = 8 * tid;
            for (; t + 24 * PICK_THREADS + 8 <= a.vocab; t += 32 * PICK_THREADS) {
                typename Of<T>::v8 v[4];
#pragma unroll
                for (int u = 0; u < 4; u++) v[u] = Of<T>::load(src + t + 8 * u * PICK_THREADS);
#pragma unroll
                for (int u = 0; u < 4; u++)
#pragma unroll
                    for (int e = 0; e < 8; e++) s += exp_of((double)v[u][e] - M);
            }
            for (; t < a.vocab; t += 8 * PICK_THREADS)
                for (int e = 0; e < 8 && t + e < a.vocab; e++) s += exp_of((double)src[t + e] - M);
            s = wave_sum(s);
            if (lane == 0) s_part[w] = s;
            __syncthreads();
            if (tid == 0) {
                s = 0.0;
                for (int q = 0; q < PICK_WAVES; q++) s += s_part[q];
                s_log[b] = log(s);
            }
            __syncthreads();
        }
        exact |= redo;
    }
    const long long o = (long long)blockIdx.x * a.n_out + tid;
    if (tid < a.n_out) {
        const bool there = tid < found;
        const Candidate c = top[there ? tid : 0];
        a.scores_out[o] = there ? (float)c.s : NONE;
        a.parent[o] = there ? (int)row0 + c.beam() : -1;
        a.token[o] = there ? c.token() : a.eos < 0 ? 0 : a.eos;
        if (a.ended_out) a.ended_out[o] = !there || s_state[c.beam()] == ENDED || c.token() == a.eos;
    }
}

// How far two scores may be from where they are known to be, together.  A sum's relative error in units of 2^-24, with p_t the softmax: an
// exponential's argument is rounded once (fp32 logits: twice), and log2 e is a quarter of a unit off: sum p_t (max - x_t) times that,
// where sum p_t (max - x_t) is the entropy less log(sum) and so at most log(vocab); v_exp_f32 2, the sum of a group of 8 3; the rest is in 64 bits.
double near_of(int vocab, bool f32) { return 2.0 / 16777216.0 * ((f32 ? 2.25 : 1.25) * std::log((double)vocab) + 6.0); }

struct Plan {
    int groups, parts;
};

// Groups of 8 logits to a thread: 8 of them (a piece of 16 384) from two workgroups a compute unit on, 4 from one, else 2.  Larger pieces
// are fewer starts and fewer picks to join, smaller ones reach more units.  us a call with 2 / 4 / 8, one box: 64 x 8 rows of 131072
// 58 / 41 / 35, 64 x 4 of 50257 21 / 17.5 / 16.4, 32 x 4 15.9 / 14.5 / 14.1, 16 x 4 11.8 / 11.4 / 11.5, 1 x 4 9.9 / 10.1 / 10.8, 8 x 8
// fp32 rows of 131072, 16 picked, 37 / 26 / 23; where one beam of eight lives, which only the device knows, the smaller are ahead: 48 x 8
// of 65024 15.4 / 16.6 / 18.0.
Plan plan(long long rows, int vocab)
{
    auto parts = [&](int g) { return (int)(((long long)vocab + 8 * THREADS * g - 1) / (8 * THREADS * g)); };
    if (rows * parts(8) >= 512) return {8, parts(8)};
    if (rows * parts(4) >= 256) return {4, parts(4)};
    return {2, parts(2)};
}

template <class T>
hipError_t launch(const BeamArgs& a, const Plan& p, Sum* sums, Pick* picks, hipStream_t st)
{
    const int keep = a.n_out;
    const unsigned grid = (unsigned)((long long)a.items * a.beams * p.parts);
    const Div parts(p.parts);
    switch (p.groups) {
    case 2: beam_scan_kernel<T, 2><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    case 4: beam_scan_kernel<T, 4><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    default: beam_scan_kernel<T, 8><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    beam_pick_kernel<T><<<(unsigned)a.items, PICK_THREADS, 0, st>>>(a, parts, Div(p.parts * keep), near_of(a.vocab, std::is_same<T, float>::value), sums, picks);
    return hipGetLastError();
}

size_t sums_bytes(long long rows, int parts) { return ((size_t)rows * parts * sizeof(Sum) + 255) & ~(size_t)255; }

}  // namespace

int beam_parts(long long rows, int vocab) { return plan(rows, vocab).parts; }

size_t beam_ws(long long rows, int vocab, int n_out)
{
    const int parts = plan(rows, vocab).parts;
    return sums_bytes(rows, parts) + (size_t)rows * parts * n_out * sizeof(Pick) + 256;
}

hipError_t launch_beam_select(const BeamArgs& a, bool f32, void* ws, hipStream_t st)
{
    const long long rows = (long long)a.items * a.beams;
    const Plan p = plan(rows, a.vocab);
    Sum* const sums = (Sum*)ws;
    Pick* const picks = (Pick*)((char*)ws + sums_bytes(rows, p.parts));
    return f32 ? launch<float>(a, p, sums, picks, st) : launch<_Float16>(a, p, sums, picks, st);
}

}  // namespace llmint8
