// beam_select: the best continuations of an item's beams, from their logits.
//
// s(b, t) = c_b + x_bt - lse_b, lse_b = log sum_t exp(x_bt).  Within a beam the order is that of the logits, which are exact; between
// beams it hangs on the lse, sums in fp32 whose error is known (NEAR below): where two beams' scores are nearer than that, the sums
// in question are made again in 64 bits.  So which tokens are picked does not hang on rounding.  Scores are c_b + ((x_bt - max) - log of
// the sum against it): beams whose logits differ by a constant tie, as they should.
//
// Two kernels.  beam_scan_kernel reads the logits once: a workgroup to a piece of a row, held in registers, gives the piece's maximum,
// its sum of exponentials, and its n_out largest logits.  beam_pick_kernel, a workgroup to an item, joins the sums and picks from the
// pieces' largest.
#include "beams.h"

#include <float.h>

#include "kv.h"

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
__device__ __forceinline__ float key_value(unsigned k)
{
    return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A value that is not above the k-th largest of the wave's 64, and not far below: the key's last LOW bits are left open.
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
    return at >= order_key(-FLT_MAX) ? key_value(at) : NONE;  // (below that: -inf, its last bits cleared)
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x = __builtin_fmaxf(x, __shfl_xor(x, d));
    return x;
}
template <class V>
__device__ __forceinline__ V wave_sum(V x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
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
    static __device__ __forceinline__ v8 load(const _Float16* p) { return __builtin_bit_cast(h8v, load8((const unsigned short*)p)); }
    static __device__ __forceinline__ float largest(v8 v)
    {
        const u4 w = __builtin_bit_cast(u4, v);
        const h2 m = __builtin_bit_cast(h2, pk_max_f16(pk_max_f16(w[0], w[1]), pk_max_f16(w[2], w[3])));
        return __builtin_fmaxf((float)m[0], (float)m[1]);
    }
};
template <>
struct Of<float> {
    typedef f8v v8;
    typedef f8v at4 __attribute__((aligned(4)));
    static __device__ __forceinline__ v8 load(const float* p) { return *(const at4*)p; }
    static __device__ __forceinline__ float largest(v8 v)
    {
        float m = v[0];
#pragma unroll
        for (int e = 1; e < 8; e++) m = __builtin_fmaxf(m, v[e]);
        return m;
    }
};

// A row's beam has logits to look at.  (NaN and +inf as a score: beam_pick_kernel tells of it.)
__device__ __forceinline__ bool lives(const BeamArgs& a, long long row)
{
    const float c = a.scores[row];
    return c > NONE && c <= FLT_MAX && !(a.ended && a.ended[row]);
}

constexpr int FEW = THREADS;  // what a piece's largest are picked from: most pieces have two to four times what they keep

// G groups of 8 logits to a thread: a wave's lanes side by side, the waves side by side, then the groups, so that a piece is
// read in runs of 4 KiB (fp16).
template <class T, int G>
__global__ void __launch_bounds__(THREADS) beam_scan_kernel(const BeamArgs a, const Div parts, int keep, float2* __restrict__ sums, Pick* __restrict__ picks)
{
    __shared__ float s_max[WAVES], s_sum[WAVES], s_tau[WAVES];
    __shared__ Pick few[FEW];
    __shared__ int s_n;
    typedef Of<T> O;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = parts.quot((int)blockIdx.x), part = (int)blockIdx.x - row * (int)parts.d;
    if (!lives(a, row)) return;
    const T* const src = (const T*)a.logits + row * a.ld;
    const int base = part * (8 * THREADS * G) + 512 * w, vocab = a.vocab;
    if (tid == 0) s_n = 0;

    typename O::v8 x[G];
    if ((part + 1) * (8ll * THREADS * G) <= vocab) {
#pragma unroll
        for (int g = 0; g < G; g++) x[g] = O::load(src + base + g * (8 * THREADS) + 8 * lane);
    } else {  // the row's last piece
#pragma unroll
        for (int g = 0; g < G; g++) {
            const long long at = (long long)base + g * (8 * THREADS);
            if (at + 512 <= vocab) {
                x[g] = O::load(src + at + 8 * lane);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) x[g][e] = (T)NONE;
                if (at < vocab) {
                    T y[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) y[e] = src[at + 8 * lane + e < vocab ? at + 8 * lane + e : vocab - 1];
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (at + 8 * lane + e < vocab) x[g][e] = y[e];
                }
            }
        }
    }

    float top[G], m = NONE;
#pragma unroll
    for (int g = 0; g < G; g++) {
        top[g] = O::largest(x[g]);
        m = __builtin_fmaxf(m, top[g]);
    }
    // (A mask of the type's lowest value is a logit like others: the reference is the maximum itself, -inf apart.)
    const float M = __builtin_fmaxf(wave_max(m), -FLT_MAX);
    float sum = 0.0f;
#pragma unroll
    for (int g = 0; g < G; g++) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = __builtin_amdgcn_exp2f(((float)x[g][e] - M) * LOG2E);
        sum += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    }
    sum = wave_sum(sum);
    const float tau_w = not_above_kth<12>(m, keep);
    if (lane == 0) s_max[w] = M, s_sum[w] = sum, s_tau[w] = tau_w;
    __syncthreads();

    // Every wave has `keep` logits that are not below its own bound: nothing below the largest bound is wanted.
    const float tau = __builtin_fmaxf(__builtin_fmaxf(s_tau[0], s_tau[1]), __builtin_fmaxf(s_tau[2], s_tau[3]));
#pragma unroll
    for (int g = 0; g < G; g++)
        if (__ballot(top[g] >= tau && top[g] > NONE)) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float v = (float)x[g][e];
                if (v >= tau && v > NONE) {
                    const int at = atomicAdd(&s_n, 1);
                    if (at < FEW) few[at] = {v, base + g * (8 * THREADS) + 8 * lane + e};
                }
            }
        }
    __syncthreads();
    int n = s_n;
    if (n > FEW) {
        // Many equal logits, or large ones side by side: each wave shows its own, group by group, best first, so that a group has at most
        // `keep` to add.
        __syncthreads();
        Best<float, int> best(keep);
#pragma unroll 1
        for (int g = 0; g < G; g++) {
            typename O::v8 y = x[0];
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
                if (!(V > best.last)) break;
                const int l = __ffsll(__ballot(v == V)) - 1;
                if (lane == l) left &= ~(1u << e);
                best.add(V, base + g * (8 * THREADS) + 8 * l + __shfl(e, l));
            }
        }
        if (lane < keep) few[w * keep + lane] = {best.v, best.at};
        n = WAVES * keep;
        __syncthreads();
    }
    const long long at = (long long)row * parts.d + part;
    const Pick mine = few[tid < n ? tid : 0];
    const bool counts = tid < n && mine.x > NONE;
    int rank = 0;
    for (int q = 0; q < n; q++) {
        const Pick o = few[q];
        rank += o.x > mine.x || (o.x == mine.x && o.t < mine.t);
    }
    if (counts && rank < keep) picks[at * keep + rank] = mine;
    const int all = __syncthreads_count(counts);
    if (tid >= all && tid < keep) picks[at * keep + tid] = {NONE, -1};
    if (tid == 0) {
        const float top4 = __builtin_fmaxf(__builtin_fmaxf(s_max[0], s_max[1]), __builtin_fmaxf(s_max[2], s_max[3]));
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < WAVES; q++) s += s_sum[q] * __builtin_amdgcn_exp2f((s_max[q] - top4) * LOG2E);
        sums[at] = {top4, s};
    }
}

// Two scores of different beams that are nearer than this are compared by sums in 64 bits.  In units of 2^-24, with p_t the softmax: an
// exponential's argument is rounded twice, sum p_t |x_t - M| (1 + 1) <= 2 log(vocab) + 2 < 45 for vocab < 2^31; v_exp_f32 2; a
// thread's sum at most 3 + 8, a wave's 6, the workgroup's 4 and its exponential's 2 + 2 |M - M'| p < 4; the rest is in 64 bits.  Below 80
// of a score's error, 160 of a difference: 1e-5.
constexpr double NEAR = 1e-5;
constexpr int SOME = 512;  // candidates that are ranked by counting

struct Candidate {
    double s;
    int b, t;
};

template <class T>
__global__ void __launch_bounds__(THREADS) beam_pick_kernel(const BeamArgs a, const Div parts, const Div per_row, const float2* __restrict__ sums,
                                                            const Pick* __restrict__ picks)
{
    constexpr int B = LLMINT8_BEAM_MAX;
    enum { DEAD, LIVE, ENDED };
    __shared__ double s_log[B], s_cum[B], s_part[WAVES];  // s_log: of the sum of exp(x - maximum)
    __shared__ float s_max[B], s_tau[WAVES];
    __shared__ int s_state[B], s_exact[B], s_redo[B], s_n, s_again;
    __shared__ Candidate some[SOME], top[B];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long row0 = (long long)blockIdx.x * a.beams;
    const double none = -__builtin_inf();

    // sums of the rows
    for (int b = w; b < a.beams; b += WAVES) {
        const long long row = row0 + b;
        const float c = a.scores[row];
        int state = a.ended && a.ended[row] ? ENDED : LIVE;
        bool bad = !(c <= FLT_MAX);  // NaN, +inf
        if (bad || c == NONE) state = DEAD;
        float M = NONE;
        double log_sum = 0.0;
        if (state == LIVE) {
            for (int q = lane; q < (int)parts.d; q += 64) M = __builtin_fmaxf(M, sums[row * parts.d + q].x);
            M = wave_max(M);
            double s = 0.0;
            for (int q = lane; q < (int)parts.d; q += 64) {
                const float2 v = sums[row * parts.d + q];
                s += (double)v.y * exp((double)v.x - (double)M);
            }
            s = wave_sum(s);
            // NaN, or +inf (whose distance to itself is NaN), anywhere in the row makes the sum NaN.  Nothing but masked tokens: 0
            if (!(s <= DBL_MAX)) bad = true;
            if (bad || s == 0.0) state = DEAD;
            log_sum = log(s);
        }
        if (lane == 0) {
            s_log[b] = log_sum, s_cum[b] = c, s_max[b] = M, s_state[b] = state, s_exact[b] = state != LIVE;
            if (bad && a.status) atomicOr(a.status, LLMINT8_BEAM_NOT_FINITE);
        }
    }
    __syncthreads();

    const int C = a.beams * (int)per_row.d;  // the pieces' largest; behind them one for each beam that has ended
    auto candidate = [&](int c) {
        Candidate r = {none, 0, 0};
        if (c < C) {
            r.b = per_row.quot(c);
            if (s_state[r.b] == LIVE) {
                const Pick p = picks[row0 * per_row.d + c];
                r.t = p.t;
                if (p.t >= 0) r.s = s_cum[r.b] + (((double)p.x - (double)s_max[r.b]) - s_log[r.b]);
            }
        } else {
            r.b = c - C, r.t = a.eos;
            if (s_state[r.b] == ENDED) r.s = s_cum[r.b];
        }
        return r;
    };
    auto place = [](const Candidate& c) { return (long long)c.b << 32 | c.t; };

    int found;
    for (;;) {
        if (tid == 0) s_n = 0, s_again = 0;
        if (tid < B) s_redo[tid] = 0;
        double m = none;
        for (int c = tid; c < C + a.beams; c += THREADS) m = __builtin_fmax(m, candidate(c).s);
        const float tau_w = not_above_kth<8>(__double2float_rd(m), a.n_out);
        if (lane == 0) s_tau[w] = tau_w;
        __syncthreads();
        // what is picked, and what it may have to be told from
        const double tau = (double)__builtin_fmaxf(__builtin_fmaxf(s_tau[0], s_tau[1]), __builtin_fmaxf(s_tau[2], s_tau[3])) - 1.01 * NEAR;
        for (int c = tid; c < C + a.beams; c += THREADS) {
            const Candidate r = candidate(c);
            if (r.s >= tau && r.s > none) {
                const int at = atomicAdd(&s_n, 1);
                if (at < SOME) some[at] = r;
            }
        }
        __syncthreads();
        int n = s_n;
        const bool many = n > SOME, all_exact = !__syncthreads_or(tid < a.beams && !s_exact[tid]);
        if (many && all_exact) {
            Best<double, long long> best(a.n_out);
            for (int c0 = 64 * w; c0 < C + a.beams; c0 += THREADS) {
                Candidate r = {none, 0, 0};
                if (c0 + lane < C + a.beams) r = candidate(c0 + lane);
                for (;;) {
                    const unsigned long long take = __ballot(r.s > none && best.takes(r.s, place(r)));
                    if (!take) break;
                    const int l = __ffsll(take) - 1;
                    best.add(__shfl(r.s, l), __shfl(place(r), l));
                    if (lane == l) r.s = none;
                }
            }
            if (lane < a.n_out) some[w * a.n_out + lane] = {best.v, (int)(best.at >> 32), (int)best.at};
            n = WAVES * a.n_out;
            __syncthreads();
        }
        found = 0;
        for (int t0 = 0; t0 < n && !(many && !all_exact); t0 += THREADS) {
            const int t = t0 + tid;
            const Candidate mine = some[t < n ? t : 0];
            const bool counts = t < n && mine.s > none;
            int rank = 0;
            for (int q = 0; q < n; q++) {
                const Candidate o = some[q];
                rank += o.s > mine.s || (o.s == mine.s && place(o) < place(mine));
            }
            if (counts && rank < a.n_out) top[rank] = mine;
            found += __syncthreads_count(counts);
        }
        found = found < a.n_out ? found : a.n_out;
        if (all_exact) break;
        if (many) {  // too many to compare them
            if (tid < a.beams && !s_exact[tid]) s_redo[tid] = 1, s_again = 1;
        } else {
            for (int t = tid; t < n; t += THREADS) {
                const Candidate q = some[t];
                for (int r = 0; r < found; r++) {
                    const Candidate p = top[r];
                    if (p.b != q.b && __builtin_fabs(p.s - q.s) < NEAR && !(s_exact[p.b] && s_exact[q.b])) {
                        s_again = 1;
                        if (!s_exact[p.b]) s_redo[p.b] = 1;
                        if (!s_exact[q.b]) s_redo[q.b] = 1;
                    }
                }
            }
        }
        __syncthreads();
        if (!s_again) break;
        for (int b = 0; b < a.beams; b++) {
            if (!s_redo[b]) continue;  // the same for all threads
            const T* const src = (const T*)a.logits + (row0 + b) * a.ld;
            const double M = s_max[b];
            double s = 0.0;
            int t = tid;
            for (; t + 7 * THREADS < a.vocab; t += 8 * THREADS) {
                T v[8];
#pragma unroll
                for (int u = 0; u < 8; u++) v[u] = src[t + u * THREADS];
#pragma unroll
                for (int u = 0; u < 8; u++) s += exp((double)v[u] - M);
            }
            for (; t < a.vocab; t += THREADS) s += exp((double)src[t] - M);
            s = wave_sum(s);
            if (lane == 0) s_part[w] = s;
            __syncthreads();
            if (tid == 0) s_log[b] = log((s_part[0] + s_part[1]) + (s_part[2] + s_part[3])), s_exact[b] = 1;
            __syncthreads();
        }
    }
    const long long o = (long long)blockIdx.x * a.n_out + tid;
    if (tid < a.n_out) {
        const bool there = tid < found;
        const Candidate c = top[there ? tid : 0];
        a.scores_out[o] = there ? (float)c.s : NONE;
        a.parent[o] = there ? (int)(row0 + c.b) : -1;
        a.token[o] = there ? c.t : a.eos < 0 ? 0 : a.eos;
        if (a.ended_out) a.ended_out[o] = !there || s_state[c.b] == ENDED || c.t == a.eos;
    }
}

struct Plan {
    int groups, parts;
};

// Logits to a thread.
Plan plan(long long rows, int vocab)
{
    auto parts = [&](int g) { return (int)(((long long)vocab + 8 * THREADS * g - 1) / (8 * THREADS * g)); };
    for (int g : {8, 4, 2})
        if (rows * parts(g) >= 1024) return {g, parts(g)};
    return {1, parts(1)};
}

template <class T>
hipError_t launch(const BeamArgs& a, const Plan& p, float2* sums, Pick* picks, hipStream_t st)
{
    const int keep = a.n_out;
    const unsigned grid = (unsigned)((long long)a.items * a.beams * p.parts);
    const Div parts(p.parts);
    switch (p.groups) {
    case 1: beam_scan_kernel<T, 1><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    case 2: beam_scan_kernel<T, 2><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    case 4: beam_scan_kernel<T, 4><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    default: beam_scan_kernel<T, 8><<<grid, THREADS, 0, st>>>(a, parts, keep, sums, picks); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    beam_pick_kernel<T><<<(unsigned)a.items, THREADS, 0, st>>>(a, parts, Div(p.parts * keep), sums, picks);
    return hipGetLastError();
}

size_t sums_bytes(long long rows, int parts) { return ((size_t)rows * parts * sizeof(float2) + 255) & ~(size_t)255; }

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
    float2* const sums = (float2*)ws;
    Pick* const picks = (Pick*)((char*)ws + sums_bytes(rows, p.parts));
    return f32 ? launch<float>(a, p, sums, picks, st) : launch<_Float16>(a, p, sums, picks, st);
}

}  // namespace llmint8
