// Attention over the 8-bit key/value cache (layout: kv.h).
//
// With codes k, v, constants c_k, c_v of a block, x_j = scale c_k / 127 (q . k_j), w_j = exp(x_j - m) / l over the positions j that
// a row sees, l = sum exp(x_j - m):  out = sum_j w_j c_v / 127 v_j.  One pass over the positions.  The values' constants go into the
// exponents: with y_j = x_j + log c_v the weight that is multiplied by a code is p_j = exp(y_j - M), M the running maximum of y, so
// that fp16 weights have their full precision where they count whatever the values' size, and a block's share of l is
// (sum p_j) / c_v.  What has been summed is scaled by exp(M_old - M_new) when M has to grow, which it need not do until weights
// get larger than some power of two (GROW, LIMIT): up to it they are as good.  Exponentials are to base 2, log2(e) being in the scale.
//
// Both products are fp16 MFMAs (32 x 32 x 16) with fp32 sums.  Codes are exact in fp16: 0x6400 + u is the fp16 number 1024 + u, so a
// byte permutation and a packed subtraction make two values of two codes.  Rows of queries are the N side of both products, S^T = K
// Q^T and O^T = V^T P^T: a lane has one row of queries, so maximum, sum and scaling need one exchange between the wave's two halves,
// and the scores a lane has computed are the operand of the second product as they are (kv.h).
//
// Roundings: a weight to fp16 (relative 2^-11, or 2^-25 of the largest), which is the operand's type and as fine as the result; l is
// summed from the fp32 weights; the fp16 values of the open block to fp16 once more, scaled by a power of two.  All sums are fp32.
#include "kv.h"

namespace llmint8 {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.0e38f;  // below every score, finite: exp2(-inf - LOWEST) is 0, where -inf - -inf would be NaN
constexpr float GROW = 8.0f;

__device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// eight codes as fp16
__device__ __forceinline__ h8 codes8(unsigned a, unsigned b)
{
    const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    a ^= 0x80808080u, b ^= 0x80808080u;
    auto two = [&](unsigned w, unsigned sel) { return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, sel)) - off; };
    const h2 p = two(a, 0x04010400u), q = two(a, 0x04030402u), r = two(b, 0x04010400u), t = two(b, 0x04030402u);
    return h8{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
}

__device__ __forceinline__ h8 pack8(const float* p)
{
    h8 r;
#pragma unroll
    for (int e = 0; e < 8; e++) r[e] = (_Float16)p[e];
    return r;
}

// What a block's scores and weights are taken by.  A block that is not there: weights of 0, by finite factors and lcv alone, since
// the constants that are read in its place may be anything, infinite ones too.
struct Factors {
    float ks;   // of the scores; above 0, so that a masked -inf stays one
    float lcv;  // log2 of the values' constant.  A block of zeros counts as 2^-24, the smallest constant: its weights count in l
    float inv;  // 1 / the values' constant
};
__device__ __forceinline__ Factors factors(bool there, float ck, float cv, float scale)
{
    cv = fmaxf(cv, 0x1p-24f);
    return {there ? fmaxf(ck * scale, 1e-30f) : 1e-30f, there ? __builtin_amdgcn_logf(cv) : -__builtin_inff(), there ? 1.0f / cv : 0.0f};
}
__device__ __forceinline__ Factors factors(bool there, unsigned c, float scale)
{
    return factors(there, f16_bits_to_float((unsigned short)(c & 0xffffu)) * (1.0f / 127.0f), f16_bits_to_float((unsigned short)(c >> 16)), scale);
}

// the larger of what the two halves of a wave hold for a row
__device__ __forceinline__ float halves_max(float x)
{
    float y = x;
    // upper half of the one with lower half of the other; two wait states behind what wrote the operands
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return fmaxf(x, y);
}

// Scores of a block of which the lane's row does not see all: those at positions outside lo .. hi - 1 out.  sc[i] is at position
// pos0 + 8 (i / 4) + 4 hh + i % 4.
__device__ __forceinline__ void hide(f16v& sc, int pos0, int hh, int lo, int hi)
{
    const int from = lo - pos0 - 4 * hh, n = hi - lo;  // of the block's positions: from .. from + n - 1
#pragma unroll
    for (int i = 0; i < 16; i++)
        if ((unsigned)(8 * (i >> 2) + (i & 3) - from) >= (unsigned)(n < 0 ? 0 : n)) sc[i] = -__builtin_inff();
}

__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float largest(const f16v& sc)
{
    float r = max3(sc[0], sc[1], sc[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) r = max3(r, sc[i], sc[i + 1]);
    return fmaxf(r, sc[15]);
}

// the largest y of a row in a block, both halves
__device__ __forceinline__ float top_of(const f16v& sc, const Factors& fa)
{
    return halves_max(fmaxf(__builtin_fmaf(largest(sc), fa.ks, fa.lcv), LOWEST));
}

// The running maximum with a block's `top`; grown(f): M grew, sums are to be scaled by f.
template <class G>
__device__ __forceinline__ void peak(float top, float& M, float& l, G grown)
{
    if (__any(top > M + GROW)) {
        const float n = fmaxf(M, top), f = exp2_(M - n);
        l *= f;
        M = n;
        grown(f);
    }
}

// Weights of a block as the operands of the second product; returns their sum, of the fp32 values, since those of a block whose
// values are small may be nothing in fp16.
__device__ __forceinline__ float expo(const f16v& sc, const Factors& fa, float M, h8 (&pf)[2])
{
    const float off = fa.lcv - M;
    float p[16], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        p[i] = exp2_(__builtin_fmaf(sc[i], fa.ks, off));
        sum += p[i];
    }
    pf[0] = pack8(p), pf[1] = pack8(p + 8);
    return sum;
}

struct AttendArgs {
    Kv kv;
    const _Float16* q;
    _Float16* out;
    long long ld_q, ld_out;
    int heads_q;
    Div group, heads;    // query heads to a key head; key heads
    float scale;         // log2(e) included
    int causal, window;
    Div splits, tiles;  // tiles: of 32 rows to a sequence, few rows
    Div units;          // workgroups to each of these
    bool by_tile;       // their order: all first tiles, all second ones, ...
    float* part;   // [split][row * heads_q + head][d] sums, not divided
    float2* stat;  // [split][row * heads_q + head] (m, l)
    bool vec;      // d and the rows of q allow 16-byte accesses
};

// Four numbers of a result: rounded in one place, since a compiler may fuse the product with the conversion (one rounding) or not (two),
// and the bits are not to hang on which store follows.
__device__ __forceinline__ h4 rounded(f4 x, float f)
{
    return h4{(_Float16)(x[0] * f), (_Float16)(x[1] * f), (_Float16)(x[2] * f), (_Float16)(x[3] * f)};
}
// those of them that a row has: the first n
__device__ __forceinline__ void put4(_Float16* dst, h4 y, int n, bool vec)
{
    if (vec) {
        if (n > 0) *(h4*)dst = y;
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < n) dst[e] = y[e];
    }
}

// features f .. f + 7 of a row of d
__device__ __forceinline__ h8 q8(const _Float16* row, int f, int d, bool vec)
{
    if (vec) return f < d ? *(const h8*)(row + f) : h8{};
    h8 r;
#pragma unroll
    for (int e = 0; e < 8; e++) r[e] = f + e < d ? row[f + e] : (_Float16)0.0f;
    return r;
}

// Operand B of the score product for one row of queries: features 32 g + 16 (lane / 32) + 8 t .. of step 2 g + t
template <int DP>
__device__ __forceinline__ void load_q(const AttendArgs& a, const KvSeq& s, int head, int r, int hh, h8 (&qf)[DP / 16])
{
    const int g = (int)a.group.d;
    if (r < s.n * g) {
        const int i = a.group.quot(r);
        const _Float16* row = a.q + (s.row0 + i) * a.ld_q + (long long)(head * g + r - i * g) * a.kv.d;
#pragma unroll
        for (int t = 0; t < DP / 16; t++) qf[t] = q8(row, 32 * (t >> 1) + 16 * hh + 8 * (t & 1), a.kv.d, a.vec);
    } else {
#pragma unroll
        for (int t = 0; t < DP / 16; t++) qf[t] = h8{};
    }
}

// Positions that a row at `pos` sees: lo .. hi - 1 (none if hi <= lo)
__device__ __forceinline__ void seen(const AttendArgs& a, int len, int pos, int& lo, int& hi)
{
    hi = !a.causal ? len : pos < 0 ? 0 : pos + 1;
    lo = a.window && pos >= a.window ? pos - a.window + 1 : 0;
}

// Blocks to a part where `blocks` are cut into at most `parts`, a multiple of `step`: not fewer than 8, so that short sequences are not
// cut into parts that cost more than they have to do
__host__ __device__ inline int chunk_of(int blocks, int parts, int step)
{
    int c = (blocks + parts - 1) / parts;
    if (parts > 1 && c < 8) c = 8;
    return (c + step - 1) / step * step;
}

// The open block's values are taken in units of this power of two, so that the largest (fp16 bits) is at most 128 of them
__device__ __forceinline__ float open_unit(unsigned largest)
{
    const unsigned b = __builtin_bit_cast(unsigned, fmaxf(f16_bits_to_float((unsigned short)largest), 0x1p-24f));
    return __builtin_bit_cast(float, (b + 0x007fffffu) & 0xff800000u) * (1.0f / 128.0f);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Few rows, or little work (kv_plan): a workgroup to a tile of 32 rows (tokens, and for each the query heads that share its keys) and a
// part of the positions.  The codes come straight into registers in operand order, every wave blocks of its own; sums meet in LDS.
// Sequences of more than 32 rows have more tiles, each of which reads and converts the blocks again: from the L2 (eight times 3 to
// 7 rows of 48 heads that share keys, 4 to 11 tiles: 1.4 times the codes come from behind it), but the conversion is about half of a
// tile's vector instructions.  Loads are marked as not to be kept, which does not keep them from the L2 for that long (the same bytes
// come from behind it without the mark), and is worth it where an axis is long (the two sequences below 91 us, 102 without).
// Single rows are bound by HBM: 1 byte a cached number, about 4 operations to it for each row, which the matrix units have to spare
// even where only one of a tile's 32 rows is there.  Each wave has two blocks on their way (of d = 128: 8 KiB each, 32 MiB on the
// chip).  Two sequences of 257 000 positions together, 64 heads over 8 of 128, one row each: 527 MB in 81 us, 6.5 TB/s (a kernel that
// only reads: 6.6 to 6.9).  64 sequences of 200 to 4 100, 32 heads over 8: 276 MB in 55 us, 5.0 TB/s; the longest sequences end last.
// Short ones are latency, from the page table to the codes to the sum of the four waves: 6.6 us for 76 positions of 12 heads of 64.
// Heads of more than 128 take 353 to 512 registers a lane, 97 to 256 of them accumulation registers: one wave to a SIMD, and 2 (of d =
// 224) or 11 (of 256) in memory.  One row over 4 000 positions of 16 heads of 256: 17 us; 64 of 200 to 4 100 of 16/2: 53.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int JOIN_FLOATS = 32 * 36;  // for a wave's sums in LDS: 32 rows of 32 features, or fewer of more

template <int DP>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2) kv_step_kernel(const AttendArgs a)
{
    constexpr int NT = DP / 32;
    __shared__ __align__(16) float s_o[4 * JOIN_FLOATS];
    __shared__ float s_m[4][32], s_l[4][32];
    const Kv& p = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), qr = lane & 31, hh = lane >> 5;
    // Workgroups go to the eight XCDs in turn: the row tiles of one part of one sequence's positions run on one XCD, one after the
    // other, and find the codes in its L2.  Or the first tiles of all parts come first (step_by_tile).
    int tile, unit;
    if (a.by_tile) {
        tile = a.units.quot(blockIdx.x), unit = a.units.rem(blockIdx.x);
    } else {
        const int turn = blockIdx.x / 8;
        tile = a.tiles.rem(turn), unit = a.tiles.quot(turn) * 8 + blockIdx.x % 8;
    }
    const int who = a.splits.quot(unit), split = a.splits.rem(unit), head = a.heads.rem(who), b = a.heads.quot(who), splits = (int)a.splits.d;
    const int g_ = (int)a.group.d;
    if (b >= p.n_seqs) return;
    KvSeq s;
    const bool ok = kv_seq(p, b, s);
    if (!ok && tid == 0) kv_flag(p, LLMINT8_KV_BAD_BATCH);
    const int r0 = 32 * tile, rows = s.n * g_ - r0 < 32 ? s.n * g_ - r0 : 32;  // this tile's
    if (rows <= 0) return;
    const int top_pos = s.len - s.n + a.group.quot(r0 + rows - 1), low_pos = s.len - s.n + a.group.quot(r0);

    // blocks that some row sees, and this workgroup's part of them
    // (lo, all_hi: of the first row; all_lo, hi: of the last.  Blocks before all_lo or behind all_hi need a mask.)
    int lo, hi, all_lo, all_hi;
    seen(a, s.len, top_pos, all_lo, hi);
    seen(a, s.len, low_pos, lo, all_hi);
    const int first = lo / KV_BLOCK, end = (hi + KV_BLOCK - 1) / KV_BLOCK;
    const int chunk = chunk_of(end - first, splits, 1);
    const int c0 = first + split * chunk, c1 = c0 + chunk < end ? c0 + chunk : end;
    const int closed = s.len / KV_BLOCK;  // blocks held as codes
    const long long total = (long long)p.n_rows * a.heads_q;
    if (split && c0 >= c1) {  // nothing left for this part
        if (tid < rows)
            a.stat[split * total + (s.row0 + a.group.quot(r0 + tid)) * (long long)a.heads_q + head * g_ + a.group.rem(r0 + tid)] = make_float2(LOWEST, 0.0f);
        return;
    }
    const int k1 = c1 < closed ? c1 : closed;

    h8 qf[DP / 16];
    int rlo, rhi;  // what this lane's row sees
    seen(a, s.len, s.len - s.n + a.group.quot(r0 + qr), rlo, rhi);

    f16v o[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) o[t] = f16v{};
    float m = LOWEST, l = 0.0f;
    auto rescale = [&](float f) {
#pragma unroll
        for (int t = 0; t < NT; t++) o[t] *= f;
    };

    // The wave's blocks: c0 + w, c0 + w + 4, ...  Lane i looks up the i-th of the next 64; two blocks are on their way at any time, a
    // block's registers being requested again as soon as they have been converted.
    const int nb = k1 > c0 + w ? (k1 - c0 - w + 3) / 4 : 0;
    struct Block {
        u4 k[NT], v[NT];
        long long at;
        Factors f;
    };
    long long at_ = 0;
    unsigned c_ = 0;
    bool there_ = false;
    Factors f_ = {};
    auto look_at = [&](int i0) {
        const int i = i0 + lane < nb ? i0 + lane : nb - 1;
        at_ = kv_block(p, b, head, c0 + w + 4 * i);
        there_ = at_ >= 0;
        if (!there_) kv_flag(p, LLMINT8_KV_BAD_PAGE);
        at_ = there_ ? at_ : 0;  // (weights of 0 for what is not there)
        c_ = p.consts[at_];
    };
    auto weigh = [&]() { f_ = factors(there_, c_, a.scale); };
    auto uniform = [](float x, int i) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i)); };
    auto place = [&](int i, Block& x) {  // the i-th block: where it is, and its factors
        x.at = (long long)__builtin_amdgcn_readlane((int)(at_ >> 32), i & 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)at_, i & 63);
    };
    auto factor = [&](int i, Block& x) { x.f = {uniform(f_.ks, i & 63), uniform(f_.lcv, i & 63), uniform(f_.inv, i & 63)}; };
    auto name = [&](int i, Block& x) {
        if ((i & 63) == 0) look_at(i), weigh();
        place(i, x), factor(i, x);
    };
    // (where: the lane; or 0, when the block is not wanted but the number of requests on their way has to be the same)
    auto request = [&](const Block& x, u4 (&y)[NT], int value, int where) {
        const u4* src = (const u4*)(p.codes + x.at * (2 * KV_BLOCK * DP)) + where + 64 * NT * value;
#pragma unroll
        for (int t = 0; t < NT; t++) y[t] = __builtin_nontemporal_load(src + 64 * t);
    };
    auto take = [&](auto refill, int i, Block& x) {
        constexpr bool REFILL = decltype(refill)::value;
        f16v sc = {};
#pragma unroll
        for (int t = 0; t < NT; t++) {
            sc = mfma(codes8(x.k[t][0], x.k[t][1]), qf[2 * t], sc);
            sc = mfma(codes8(x.k[t][2], x.k[t][3]), qf[2 * t + 1], sc);
        }
        const Factors fa = x.f;
        const int where = i + 2 < nb ? lane : 0;
        if (REFILL) {
            if (i + 2 < nb) name(i + 2, x);
            request(x, x.k, 0, where);
        }
        const int pos0 = (c0 + w + 4 * i) * KV_BLOCK;
        h8 pf[2];
        if (pos0 < all_lo || pos0 + KV_BLOCK > all_hi) hide(sc, pos0, hh, rlo, rhi);
        peak(top_of(sc, fa), m, l, rescale);
        l = __builtin_fmaf(expo(sc, fa, m, pf), fa.inv, l);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            o[t] = mfma(codes8(x.v[t][0], x.v[t][1]), pf[0], o[t]);
            o[t] = mfma(codes8(x.v[t][2], x.v[t][3]), pf[1], o[t]);
        }
        if (REFILL) request(x, x.v, 1, where);
    };
    Block x, y;
    if (nb > 0) {
        look_at(0);
        place(0, x), place(nb > 1, y);
        request(x, x.k, 0, lane), request(x, x.v, 1, lane);
        request(y, y.k, 0, nb > 1 ? lane : 0), request(y, y.v, 1, nb > 1 ? lane : 0);
    }
    load_q<DP>(a, s, head, r0 + qr, hh, qf);
    // (a wait for the rows of queries inside the loop would be one for what was requested since, too)
#pragma unroll
    for (int t = 0; t < DP / 16; t++) asm volatile("" : "+v"(qf[t]));
    if (nb > 0) {
        weigh();
        factor(0, x), factor(nb > 1, y);
        int i = 0;
        for (; i + 1 < nb; i += 2) take(std::true_type(), i, x), take(std::true_type(), i + 1, y);
        if (i < nb) take(std::false_type(), i, x);
    }
    // The open block, fp16: by the wave whose turn it is.  Its values are scaled by a power of two to what codes are, at most 128.
    if (closed >= c0 && closed < c1 && ((closed - c0) & 3) == w) {
        const int d = p.d, base = closed * KV_BLOCK;
        f16v sc = {};
        const bool there = base + qr < s.len;
        const _Float16* row = (const _Float16*)kv_ring_row(p, s.slot, head, 0, base + qr);
#pragma unroll
        for (int t = 0; t < DP / 16; t++)
            sc = mfma(there ? q8(row, 32 * (t >> 1) + 16 * hh + 8 * (t & 1), d, d % 8 == 0) : h8{}, qf[t], sc);
        unsigned short v[NT][16], big = 0;
        const unsigned short* vals = kv_ring_row(p, s.slot, head, 1, base);
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int r = 8 * (i >> 2) + 4 * hh + (i & 3), f = 32 * t + qr;
                v[t][i] = base + r < s.len && f < d ? vals[r * d + f] : (unsigned short)0;
                const unsigned short y = v[t][i] & 0x7fffu;
                big = y > big ? y : big;
            }
        int top = big;
#pragma unroll
        for (int x = 32; x; x >>= 1) {
            const int y = __shfl_xor(top, x);
            top = y > top ? y : top;
        }
        const float unit = open_unit(top);
        const Factors fa = factors(true, 1.0f, 127.0f * unit, a.scale);
        h8 pf[2];
        hide(sc, base, hh, rlo, rhi);
        peak(top_of(sc, fa), m, l, rescale);
        l = __builtin_fmaf(expo(sc, fa, m, pf), fa.inv, l);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; i++) y[i] = f16_bits_to_float(v[t][i]) * (1.0f / unit);
            o[t] = mfma(pack8(y), pf[0], o[t]);
            o[t] = mfma(pack8(y + 8), pf[1], o[t]);
        }
    }

    // ---- join the four waves
    l += __shfl_xor(l, 32);
    if (hh == 0) s_m[w][qr] = m, s_l[w][qr] = l;
    __syncthreads();
    {
        const float top = fmaxf(fmaxf(s_m[0][qr], s_m[1][qr]), fmaxf(s_m[2][qr], s_m[3][qr]));
        rescale(exp2_(m - top) * (1.0f / 127.0f));
    }
    // as many tiles of 32 features at a time as LDS has room for; rows are 4 floats longer than their data, for the banks
    const int fit = (JOIN_FLOATS / rows - 4) / 32, nt = fit < NT ? fit : NT, pitch = 32 * nt + 4;
    for (int t0 = 0; t0 < NT; t0 += nt) {
        if (t0) __syncthreads();
        if (qr < rows)
#pragma unroll
            for (int t = 0; t < NT; t++)
                if (t >= t0 && t < t0 + nt)
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        *(f4*)(s_o + (w * rows + qr) * pitch + 32 * (t - t0) + 8 * j + 4 * hh) =
                            f4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
        __syncthreads();
        const int quads = 8 * nt;  // of features
        for (int x = tid; x < quads * rows; x += 256) {
            const int f = 4 * (x % quads), r = x / quads, at = 32 * t0 + f;
            if (at >= p.d) continue;
            const float top = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
            f4 sum = {};
            float den = 0.0f;
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const f4 y = *(const f4*)(s_o + (q * rows + r) * pitch + f);
#pragma unroll
                for (int e = 0; e < 4; e++) sum[e] += y[e];
                den += s_l[q][r] * exp2_(s_m[q][r] - top);
            }
            const long long row = s.row0 + a.group.quot(r0 + r);
            const int g = head * g_ + a.group.rem(r0 + r);
            const float inv = den != 0.0f ? 1.0f / den : 0.0f;
            if (splits > 1) {
                const long long at_row = split * total + row * a.heads_q + g;
                if (at == 0) a.stat[at_row] = make_float2(top, den);
                float* dst = a.part + at_row * p.d + at;
                if (p.d % 4 == 0) {
                    *(f4*)dst = sum;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (at + e < p.d) dst[e] = sum[e];
                }
            } else {
                put4(a.out + row * a.ld_out + (long long)g * p.d + at, rounded(sum, inv), p.d - at, a.vec);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// Many rows: a workgroup takes a tile of 32 rows a wave (tokens, and for each the query heads that share its keys), its waves the
// same blocks of the cache two at a time (a stage) from LDS, where the codes lie as fp16 in operand order: they are converted once
// for all rows.  Bound by the matrix units, by what makes scores weights and by the reads of LDS, each about half of the time and
// kept busy at the same time: the scores of the next block are computed while the weights of this one are.  So LDS holds keys one
// block ahead of values.  (Operands of 64 rows a wave halve the reads, but leave one wave to a SIMD, which then issues vector
// instructions half as often: no faster.)  8 192 tokens of 40 heads of 128, each seeing those before it: 690 us, 0.99 PFLOP/s of what
// they see (675 to 730 from card to card, by the clock that power leaves); a matrix product of 16 384 x 16 384 x 16 384 by the library reaches
// 1.32.  1 024 tokens behind 20 011, 32 heads over 8: 336 us with the join, 1.02 PFLOP/s.  2 048 tokens of 32 heads: 57 us, 0.60; the
// last tile's 64 blocks are its time.  Heads of more than 128 take 356 to 512 registers: one wave to a SIMD, and 7 (of 256) in memory.
// 2 048 tokens of 16 heads of 256: 101 us, 0.34 PFLOP/s; 8 192 of 16/2: 751, 0.73.
// ---------------------------------------------------------------------------------------------------------------------------
//
// PARTS 2: two such groups of waves to a workgroup and tile, each with half of its blocks and an LDS of its own; the second's sums go to
// the first through LDS.  They meet at the same barriers, so both go through the first's number of stages (which has not fewer).
template <int DP, int WAVES, int PARTS>
__global__ void __launch_bounds__(64 * WAVES * PARTS, WAVES * PARTS == 4 && DP <= 128 ? 2 : 1) kv_prompt_kernel(const AttendArgs a)
{
    constexpr int NT = DP / 32, ROWS = 32 * WAVES, THREADS = 64 * WAVES;
    constexpr int PIECES = DP * 4, PER = (PIECES + THREADS - 1) / THREADS;  // 16-byte pieces of two blocks' keys, or values; to a thread
    extern __shared__ __align__(16) _Float16 all_lds[];                     // [PARTS][keys, values][4 blocks][DP * 32]
    __shared__ int s_big[WAVES];
    const Kv& p = a.kv;
    const int part = PARTS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    const int tid = threadIdx.x - part * THREADS, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), qr = lane & 31, hh = lane >> 5;
    _Float16* const lds = all_lds + part * 8 * DP * 32;
    // the heads of a tile one after the other: with a multiple of 8 heads, a head's tiles all run on one XCD and share its L2
    const int head = a.heads.rem(blockIdx.x), split = blockIdx.y, splits = (int)a.splits.d, G = (int)a.group.d;
    bool wrong = false;
    int b, tile;
    KvSeq s;
    const bool found = kv_find(p, a.heads.quot(blockIdx.x), [&](const KvSeq& t) { return (t.n * G + ROWS - 1) / ROWS; }, b, s, tile, wrong);
    if (wrong) kv_flag(p, LLMINT8_KV_BAD_BATCH);
    if (!found) return;
    const int rows = s.n * G, old = s.len - s.n;
    tile = (rows + ROWS - 1) / ROWS - 1 - tile;  // those that see most first
    const int r0 = tile * ROWS, r1 = r0 + ROWS < rows ? r0 + ROWS : rows;
    const int w0 = r0 + w * 32, w1 = w0 + 32 < r1 ? w0 + 32 : r1;  // this wave's rows

    int lo, hi, x0, x1;
    seen(a, s.len, old + a.group.quot(r0), lo, x1);
    seen(a, s.len, old + a.group.quot(r1 - 1), x0, hi);
    const int first = lo / KV_BLOCK, end = (hi + KV_BLOCK - 1) / KV_BLOCK;
    const int chunk = chunk_of(end - first, splits * PARTS, 2);
    const int g0 = first + split * PARTS * chunk, g1 = g0 + PARTS * chunk < end ? g0 + PARTS * chunk : end;  // the workgroup's blocks
    const int c0 = g0 + part * chunk, c1 = c0 + chunk < end ? c0 + chunk : end;                              // this part's
    const int closed = s.len / KV_BLOCK, k1 = c1 < closed ? c1 : closed;
    // (an even number of stages, so that a stage's registers are known to the compiler; one that is not there has no weights)
    const int last = g0 + chunk < closed && g0 + chunk < end ? g0 + chunk : closed < end ? closed : end;  // of the first part
    const int stages = last > g0 ? (last - g0 + 3) / 4 * 2 : 0;
    const long long total = (long long)p.n_rows * a.heads_q;
    if (split && g0 >= g1) {  // nothing left
        for (int r = r0 + (int)threadIdx.x; r < r1; r += THREADS * PARTS)
            a.stat[split * total + (s.row0 + a.group.quot(r)) * (long long)a.heads_q + head * G + a.group.rem(r)] = make_float2(LOWEST, 0.0f);
        return;
    }
    // what all of the wave's rows see, and the stages in which some see anything
    int some_lo = 0, some_hi = 0, all_lo = 0, all_hi = 0;
    if (w0 < w1) {
        seen(a, s.len, old + a.group.quot(w0), some_lo, all_hi);
        seen(a, s.len, old + a.group.quot(w1 - 1), all_lo, some_hi);
    }
    auto clip = [&](int x) { return x < 0 ? 0 : x > stages ? stages : x; };
    const int sa = clip((some_lo / KV_BLOCK - c0) >> 2 << 1), sb = clip(((some_hi + KV_BLOCK - 1) / KV_BLOCK - c0 + 3) >> 2 << 1);

    // ---- Lane i of every wave looks up the i-th of 64 blocks, so that a stage waits neither for the page table nor for constants.
    // `ahead` are 64 blocks from PERIOD behind the first of those in use on.
    constexpr int PERIOD = 56;
    struct Looked {
        int at[2];  // where a block's codes begin
        unsigned c;
        bool there;
        Factors f;
    };
    auto look_at = [&](int j) {
        Looked r;
        const int k = c0 + j + lane;
        long long at = kv_block(p, b, head, k < k1 ? k : k1 - 1);
        if (at < 0) kv_flag(p, LLMINT8_KV_BAD_PAGE);
        r.there = at >= 0 && k < k1;
        at = at < 0 ? 0 : at;  // (weights of 0 for what is not there)
        r.c = p.consts[at];
        at *= 2 * KV_BLOCK * DP;
        r.at[0] = (int)at, r.at[1] = (int)(at >> 32);
        return r;
    };
    auto look_up = [&](int j) {
        Looked r = look_at(j);
        r.f = factors(r.there, r.c, a.scale);
        return r;
    };
    Looked use, ahead;
    int j0 = 0;  // the first block of `use`
    auto float_at = [&](float x, int j) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), j - j0)); };
    auto factors_of = [&](int j) { return Factors{float_at(use.f.ks, j), float_at(use.f.lcv, j), float_at(use.f.inv, j)}; };
    // where the keys and values of block j lie in LDS, by j % 4 (a constant wherever it matters)
    h8* const my_lds = (h8*)lds + lane;
    auto keys = [&](int j) { return my_lds + (j & 3) * (DP * 4); };
    auto values = [&](int j) { return my_lds + (4 + (j & 3)) * (DP * 4); };
    // this thread's 16-byte pieces of the keys (value 0) or values of blocks j and j + 1
    auto request = [&](int j, int value, u4 (&piece)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int t = w * 64 + THREADS * i, x = t >= DP * 2, u = t - x * DP * 2;  // a wave's pieces are of one block
            if (PIECES % THREADS && t >= PIECES) break;
            const long long at = (long long)__builtin_amdgcn_readlane(use.at[1], j + x - j0) << 32 |
                                 (unsigned)__builtin_amdgcn_readlane(use.at[0], j + x - j0);
            piece[i] = *((const u4*)(p.codes + at) + value * DP * 2 + u + lane);
        }
    };
    // the i-th of them into LDS, converted: its first or second eight codes
    auto deposit_half = [&](int j, int value, const u4& piece, int i, int half) {
        const int t = w * 64 + THREADS * i, x = t >= DP * 2, u = t - x * DP * 2;
        if (PIECES % THREADS && t >= PIECES) return;
        ((value ? values(j + x) : keys(j + x)) + 2 * u)[64 * half] = codes8(piece[2 * half], piece[2 * half + 1]);
    };
    auto deposit = [&](int j, int value, const u4 (&piece)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; i++) deposit_half(j, value, piece[i], i, 0), deposit_half(j, value, piece[i], i, 1);
    };

    // what the first stages need is requested before the rows of queries are
    struct Pieces {
        u4 k[PER], v[PER];
    };
    Pieces first_, even, odd;  // what is on its way for stages of even and odd numbers: two stages ahead, the latency of a load
    u4 k1_[PER];
    if (stages) {
        use = look_at(0);  // (what is requested next does not wait for the constants)
        request(0, 0, first_.k), request(1, 0, k1_), request(0, 1, first_.v);
        request(3, 0, even.k), request(2, 1, even.v), request(5, 0, odd.k), request(4, 1, odd.v);
    }
    h8 qf[DP / 16];
    load_q<DP>(a, s, head, w0 + qr, hh, qf);
    int rlo, rhi;
    seen(a, s.len, old + a.group.quot(w0 + qr), rlo, rhi);
    const int full_hi = rhi < s.len ? rhi : s.len;
    if (rhi > k1 * KV_BLOCK) rhi = k1 * KV_BLOCK;  // behind that there is nothing of this workgroup's but the open block
    if (all_hi > k1 * KV_BLOCK) all_hi = k1 * KV_BLOCK;
    f16v o[NT];
    float m = LOWEST, l = 0.0f;
#pragma unroll
    for (int x = 0; x < NT; x++) o[x] = f16v{};
    auto rescale = [&](float x) {
#pragma unroll
        for (int q = 0; q < NT; q++) o[q] *= x;
    };
    auto scores = [&](int j, f16v& sc) {
        const h8* const kb = keys(j);
        sc = f16v{};
#pragma unroll
        for (int g = 0; g < DP / 16; g++) sc = mfma(kb[g * 64], qf[g], sc);
    };

    // Block j, whose scores are sc and whose first eight weights a lane are there (pfa, their sum suma): the next block's scores,
    // product by product, and between these products the other eight weights; then the block's sums, and between these products the next
    // block's first eight weights.  So the matrix unit and the vector unit have the same share of each slice, which is what keeps
    // both busy with the two waves to a SIMD that registers allow.  other(x), x = 0 .. 7: an eighth of what else there is to do.
    // The order is fixed slice by slice: operands are read from LDS some slices ahead (its latency) and no further, or registers run
    // out.  k: the next block's first keys; on return, if NEXT, those of the one behind.
    //
    // No maximum is taken: M stays as it is unless a weight sum says that it is too low (above LIMIT, which fp16 weights up to that
    // stand; infinite where a row has seen nothing yet), and then the block's weights are made anew.
    constexpr int S = DP / 16, AHEAD = S < 4 ? S : 4, U = 2 * NT;
    constexpr float LIMIT = 4096.0f;
    h8 pfa;
    float suma;
    auto first_keys = [&](int j, h8 (&k)[AHEAD]) {
        const h8* const kb = keys(j);
#pragma unroll
        for (int g = 0; g < AHEAD; g++) k[g] = kb[g * 64];
    };
    auto masked = [&](int j, f16v& sc) {
        const int pos0 = (c0 + j) * KV_BLOCK;
        if (pos0 < all_lo || pos0 + KV_BLOCK > all_hi) hide(sc, pos0, hh, rlo, rhi);
    };
    auto step = [&](auto slot, auto with_next, int j, const f16v& sc, const Factors& fa, f16v& next, const Factors& fb, h8 (&k)[AHEAD],
                    auto other) {
        constexpr int J = decltype(slot)::value;  // j % 4
        constexpr bool NEXT = decltype(with_next)::value;
        const h8 *const kb = keys(J + 1), *const kc = keys(J + 2), *const vb = values(J);
        float off = fa.lcv - m, sum = suma, p[8];
        h8 pf[2], v[NT];
        pf[0] = pfa;
        next = f16v{};
#pragma unroll
        for (int g = 0; g < S; g++) {
            const h8 t = k[g % AHEAD];
            if (g + AHEAD < S) k[g % AHEAD] = kb[(g + AHEAD) * 64];
#pragma unroll
            for (int q = 0; q < NT; q++)  // the values' first operands over the last slices
                if (g == S - AHEAD + q * AHEAD / NT) v[q] = vb[2 * q * 64];
            next = mfma(t, qf[g], next);
#pragma unroll
            for (int i = 8 * g / S; i < 8 * (g + 1) / S; i++) {
                p[i] = exp2_(__builtin_fmaf(sc[8 + i], fa.ks, off));
                if (i & 1) pf[1][i - 1] = (_Float16)p[i - 1], pf[1][i] = (_Float16)p[i];
                if (i) sum += p[i - 1];
            }
#pragma unroll
            for (int x = 0; x < 4; x++)
                if (g == x * S / 4) other(x);
            __builtin_amdgcn_sched_barrier(0);
        }
        sum += p[7];
        if (__any(sum > LIMIT)) {
            const float n = fmaxf(m, top_of(sc, fa)), f = exp2_(m - n);
            l *= f;
            m = n;
            rescale(f);
            sum = expo(sc, fa, m, pf);
        }
        l = __builtin_fmaf(sum, fa.inv, l);
        masked(j + 1, next);
        off = fb.lcv - m;
        suma = 0.0f;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int y = u / NT, q = u % NT;
            const h8 t = v[q];
            if (y == 0) v[q] = vb[(2 * q + 1) * 64];
            if (NEXT && y == 1)
#pragma unroll
                for (int g = 0; g < AHEAD; g++)
                    if (g * NT / AHEAD == q) k[g] = kc[g * 64];
            o[q] = mfma(t, pf[y], o[q]);
            if (u)  // (the last product of the scores takes a while)
#pragma unroll
                for (int i = 8 * (u - 1) / (U - 1); i < 8 * u / (U - 1); i++) {
                    p[i] = exp2_(__builtin_fmaf(next[i], fb.ks, off));
                    if (i & 1) pfa[i - 1] = (_Float16)p[i - 1], pfa[i] = (_Float16)p[i];
                    if (i) suma += p[i - 1];
                }
#pragma unroll
            for (int x = 0; x < 4; x++)
                if (u == x * U / 4) other(4 + x);
            __builtin_amdgcn_sched_barrier(0);
        }
        suma += p[7];
    };

    // ---- the open block, fp16 from the ring, before the others
    if (closed >= g0 && closed < g1) {
        const bool mine = closed >= c0 && closed < c1;
        const int d = p.d, pos0 = closed * KV_BLOCK;
        const unsigned short *const krows = kv_ring_row(p, s.slot, head, 0, pos0), *const vrows = kv_ring_row(p, s.slot, head, 1, pos0);
        int big = 0;
        if (mine) {
            for (int t = tid; t < (s.len - pos0) * d; t += THREADS) {
                const int y = vrows[t] & 0x7fff;
                big = y > big ? y : big;
            }
#pragma unroll
            for (int x = 32; x; x >>= 1) {
                const int y = __shfl_xor(big, x);
                big = y > big ? y : big;
            }
            if (lane == 0) s_big[w] = big;
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < WAVES; x++) big = s_big[x] > big ? s_big[x] : big;
        const float unit = open_unit(big);
        if (mine)
            for (int t = tid; t < KV_BLOCK * DP / 8; t += THREADS) {  // eight of a lane's keys and values each
                const int at = t >> 6, r = t & 31, h = (t >> 5) & 1, f = 32 * (at >> 1) + r;
                h8 y = {}, z = {};
                if (pos0 + r < s.len) y = q8((const _Float16*)krows + r * d, 32 * (at >> 1) + 16 * h + 8 * (at & 1), d, d % 8 == 0);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int q = 16 * (at & 1) + 8 * (i >> 2) + 4 * h + (i & 3);
                    if (pos0 + q < s.len && f < d) z[i] = (_Float16)(f16_bits_to_float(vrows[q * d + f]) * (1.0f / unit));
                }
                *((h8*)lds + t) = y;
                *((h8*)(lds + 4 * DP * 32) + t) = z;
            }
        __syncthreads();
        if (mine && pos0 < some_hi) {
            f16v sc;
            scores(0, sc);
            const Factors fa = factors(true, 1.0f, 127.0f * unit, a.scale);
            hide(sc, pos0, hh, rlo, full_hi);
            peak(top_of(sc, fa), m, l, rescale);
            h8 pf[2];
            l = __builtin_fmaf(expo(sc, fa, m, pf), fa.inv, l);
            const h8* const vb = values(0);
#pragma unroll
            for (int y = 0; y < 2; y++)
#pragma unroll
                for (int q = 0; q < NT; q++) o[q] = mfma(vb[(2 * q + y) * 64], pf[y], o[q]);
        }
        __syncthreads();
    }

    // ---- Stage st: blocks 2 st and 2 st + 1 (from c0 on): their weights and sums, and each time the scores of the block behind.  So keys
    // go to LDS one block earlier than values: meanwhile those of 2 st + 3 and 2 st + 4, and the values of 2 st + 2 and 2 st + 3.
    if (stages) {
        use.f = factors(use.there, use.c, a.scale);
        ahead = use;  // (its addresses may be read from once more after the last block)
        if (k1 - c0 > PERIOD) ahead = look_up(PERIOD);
        deposit(0, 0, first_.k);
        __syncthreads();  // (block 1's keys come twice)
        deposit(1, 0, k1_), deposit(0, 1, first_.v);
        __syncthreads();
        auto more = [&](int st, Pieces& x) {  // the end of a stage
            if (2 * st + 2 == j0 + PERIOD) {
                use = ahead, j0 += PERIOD;
                if (k1 - c0 > j0 + PERIOD) ahead = look_up(j0 + PERIOD);
            }
            request(2 * st + 7, 0, x.k), request(2 * st + 6, 1, x.v);
            __syncthreads();
        };
        // The wave's first scores are computed in the stage before (its keys are overwritten in its own)
        f16v s0, s1;
        Factors f0;
        auto enter = [&]() {
            scores(2 * sa, s0);
            f0 = factors_of(2 * sa);
            masked(2 * sa, s0);
            h8 pf[2];
            expo(s0, f0, m, pf);
            pfa = pf[0];
            suma = __builtin_inff();  // (the weights are made anew by M's first value if a row has none, and by any other)
        };
        auto idle = [&](int st, Pieces& x) {  // a stage in which the wave's rows see nothing
            deposit(2 * st + 3, 0, x.k), deposit(2 * st + 2, 1, x.v);
            more(st, x);
        };
        auto busy = [&](auto slot, int st, Pieces& x) {
            constexpr int J = decltype(slot)::value;
            typedef std::integral_constant<int, J> first;
            typedef std::integral_constant<int, J + 1> second;
            h8 k[AHEAD];
            first_keys(J + 1, k);
            const Factors f1 = factors_of(2 * st + 1);
            // the conversions: keys in the first half of the stage, values in the second, and not before what they come from is there
            auto part = [&](int value, const u4 (&y)[PER], int n) {
#pragma unroll
                for (int i = 0; i < 2 * PER; i++)
                    if (n == (8 * i + 4) / (2 * PER)) deposit_half(value ? J + 2 : J + 3, value, y[i >> 1], i >> 1, i & 1);
            };
            step(first(), std::true_type(), 2 * st, s0, f0, s1, f1, k, [&](int n) { part(0, x.k, n); });
            f0 = factors_of(2 * st + 2);
            step(second(), std::false_type(), 2 * st + 1, s1, f1, s0, f0, k, [&](int n) { part(1, x.v, n); });
            more(st, x);
        };
        // The rows of queries have to be there before the loop: a wait for them inside would be one for what was requested since, too
#pragma unroll
        for (int t = 0; t < DP / 16; t++) asm volatile("" : "+v"(qf[t]));
        if (sa == 0) enter();
        __syncthreads();
        int st = 0;
        for (; st < sa; st += 2) {
            idle(st, even);
            if (st + 2 == sa) enter();
            idle(st + 1, odd);
        }
        for (; st < sb; st += 2) busy(std::integral_constant<int, 0>(), st, even), busy(std::integral_constant<int, 2>(), st + 1, odd);
        for (; st < stages; st += 2) idle(st, even), idle(st + 1, odd);
    }

    if constexpr (PARTS == 2) {
        f4* const sums = (f4*)all_lds + w * NT * 4 * 64 + lane;
        float2* const stat = (float2*)((f4*)all_lds + WAVES * NT * 4 * 64) + w * 64 + lane;
        __syncthreads();  // (the last stage's operands have been read)
        if (part) {
            *stat = make_float2(m, l);
#pragma unroll
            for (int q = 0; q < NT; q++)
#pragma unroll
                for (int j = 0; j < 4; j++) sums[(q * 4 + j) * 64] = f4{o[q][4 * j], o[q][4 * j + 1], o[q][4 * j + 2], o[q][4 * j + 3]};
        }
        __syncthreads();
        if (part) return;
        const float2 t = *stat;
        const float top = fmaxf(m, t.x), f = exp2_(m - top), g = exp2_(t.x - top);
        m = top, l = l * f + t.y * g;
#pragma unroll
        for (int q = 0; q < NT; q++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const f4 y = sums[(q * 4 + j) * 64];
#pragma unroll
                for (int e = 0; e < 4; e++) o[q][4 * j + e] = o[q][4 * j + e] * f + y[e] * g;
            }
    }
    const float den = l + __shfl_xor(l, 32);
    const int r = w0 + qr;
    if (r >= r1) return;
    const long long row = s.row0 + a.group.quot(r);
    const int g = head * G + a.group.rem(r);
    if (splits > 1) {
        const long long at = split * total + row * a.heads_q + g;
        if (hh == 0) a.stat[at] = make_float2(m, den);
        float* dst = a.part + at * p.d;
#pragma unroll
        for (int q = 0; q < NT; q++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int f = 32 * q + 8 * j + 4 * hh;
                const float u = 1.0f / 127.0f;
                const f4 y = {o[q][4 * j] * u, o[q][4 * j + 1] * u, o[q][4 * j + 2] * u, o[q][4 * j + 3] * u};
                if (p.d % 4 == 0) {
                    if (f < p.d) *(f4*)(dst + f) = y;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (f + e < p.d) dst[f + e] = y[e];
                }
            }
    } else {
        _Float16* dst = a.out + row * a.ld_out + (long long)g * p.d;
        const float inv = den != 0.0f ? (1.0f / 127.0f) / den : 0.0f;
#pragma unroll
        for (int q = 0; q < NT; q++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int f = 32 * q + 8 * j + 4 * hh;
                put4(dst + f, rounded(f4{o[q][4 * j], o[q][4 * j + 1], o[q][4 * j + 2], o[q][4 * j + 3]}, inv), p.d - f, a.vec);
            }
    }
}

// Joins the splits, many of them: four waves to a row and head, 16 lanes x 4 features (as many times as d has them) to a split, the
// splits dealt out over the waves and their quarters, four in flight each.  A part that had nothing to do has l = 0, and its sums
// were not written.  Latency: 4.8 us for 128 rows and heads in 32 parts.
__global__ void __launch_bounds__(256) kv_join_kernel(const AttendArgs a)
{
    const int splits = (int)a.splits.d;
    constexpr int NQ = KV_MAX_D / 64;
    __shared__ f4 s_sum[4][NQ][16];
    __shared__ float s_den[4];
    const int tid = threadIdx.x, lane = tid & 63, d = a.kv.d, w = tid >> 6;
    const long long total = (long long)a.kv.n_rows * a.heads_q, x = blockIdx.x;
    float top = LOWEST;
    for (int s = lane; s < splits; s += 64) {
        const float2 t = a.stat[s * total + x];
        if (t.y != 0.0f) top = fmaxf(top, t.x);
    }
#pragma unroll
    for (int y = 32; y; y >>= 1) top = fmaxf(top, __shfl_xor(top, y));
    const int part = lane >> 4, f0 = 4 * (lane & 15);
    f4 sum[NQ] = {};
    float den = 0.0f;
    for (int s0 = 4 * w + part; s0 < splits; s0 += 64) {
        f4 v[4][NQ];
        float f[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int s = s0 + 16 * u;
            const bool there = s < splits;
            const float2 t = there ? a.stat[s * total + x] : make_float2(0.0f, 0.0f);
            const float* src = a.part + (s * total + x) * d + f0;
            f[u] = t.y != 0.0f ? exp2_(t.x - top) : 0.0f;
            den += f[u] * t.y;
#pragma unroll
            for (int q = 0; q < NQ; q++) {
                v[u][q] = f4{};
                if (there && f0 + 64 * q < d) {
                    if (d % 4 == 0) {
                        v[u][q] = *(const f4*)(src + 64 * q);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (f0 + 64 * q + e < d) v[u][q][e] = src[64 * q + e];
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
            if (f[u] != 0.0f)
#pragma unroll
                for (int q = 0; q < NQ; q++)
#pragma unroll
                    for (int e = 0; e < 4; e++) sum[q][e] += f[u] * v[u][q][e];
    }
#pragma unroll
    for (int y = 16; y < 64; y <<= 1) {
        den += __shfl_xor(den, y);
#pragma unroll
        for (int q = 0; q < NQ; q++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[q][e] += __shfl_xor(sum[q][e], y);
    }
    if (lane < 16)
#pragma unroll
        for (int q = 0; q < NQ; q++) s_sum[w][q][lane] = sum[q];
    if (lane == 0) s_den[w] = den;
    __syncthreads();
    if (w || lane >= 16) return;
    den = s_den[0] + s_den[1] + s_den[2] + s_den[3];
    _Float16* dst = a.out + x / a.heads_q * a.ld_out + x % a.heads_q * d + f0;
#pragma unroll
    for (int q = 0; q < NQ; q++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float y = s_sum[0][q][lane][e] + s_sum[1][q][lane][e] + s_sum[2][q][lane][e] + s_sum[3][q][lane][e];
            if (f0 + 64 * q + e < d) dst[64 * q + e] = (_Float16)(den != 0.0f ? y / den : 0.0f);
        }
}

// The same for at most N: a thread to four features of a row and head, everything requested at once (40 rows and heads in 12 parts:
// 3.9 us against 4.2, 1 920 in 10: 4.7 against 10).  HBM where rows are many: 1 024 rows of 32 heads in two parts, 9.3 us (12.7 where N is
// 16).
template <int N>
__global__ void __launch_bounds__(256) kv_join_few_kernel(const AttendArgs a)
{
    const int splits = (int)a.splits.d;
    const int d = a.kv.d, quads = (d + 3) / 4;
    const long long total = (long long)a.kv.n_rows * a.heads_q, t = (long long)blockIdx.x * 256 + threadIdx.x, x = t / quads;
    if (x >= total) return;
    const int f0 = 4 * (int)(t - x * quads);
    float2 st[N];
    f4 v[N];
#pragma unroll
    for (int s = 0; s < N; s++) {
        st[s] = s < splits ? a.stat[s * total + x] : make_float2(LOWEST, 0.0f);
        v[s] = f4{};
        if (s < splits) {
            const float* src = a.part + (s * total + x) * d + f0;
            if (d % 4 == 0) {
                v[s] = *(const f4*)src;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (f0 + e < d) v[s][e] = src[e];
            }
        }
    }
    float top = LOWEST, den = 0.0f;
#pragma unroll
    for (int s = 0; s < N; s++)
        if (st[s].y != 0.0f) top = fmaxf(top, st[s].x);
    f4 sum = {};
#pragma unroll
    for (int s = 0; s < N; s++)
        if (st[s].y != 0.0f) {
            const float f = exp2_(st[s].x - top);
            den += f * st[s].y;
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += f * v[s][e];
        }
    const float inv = den != 0.0f ? 1.0f / den : 0.0f;
    _Float16* dst = a.out + x / a.heads_q * a.ld_out + x % a.heads_q * d + f0;
    put4(dst, rounded(sum, inv), d - f0, a.vec);
}

template <int DP>
hipError_t launch_step(const AttendArgs& a, const KvPlan& plan, hipStream_t st)
{
    kv_step_kernel<DP><<<(unsigned)kv_attention_workgroups(a.kv, plan), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DP, int WAVES, int PARTS>
hipError_t launch_prompt(const AttendArgs& a, int tiles, hipStream_t st)
{
    constexpr int bytes = PARTS * 8 * DP * 32 * 2;
    if (bytes + 256 > 65536) {  // with the static part
        const hipError_t e = hipFuncSetAttribute((const void*)kv_prompt_kernel<DP, WAVES, PARTS>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    kv_prompt_kernel<DP, WAVES, PARTS><<<dim3(tiles * a.kv.heads, a.splits.d), 64 * WAVES * PARTS, bytes, st>>>(a);
    return hipGetLastError();
}

}  // namespace

constexpr int KV_STEP_ROWS = 32;

KvPlan kv_plan(const Kv& p, int heads_q, int window)
{
    KvPlan r = {};
    const long long group = heads_q / p.heads, rows = p.max_rows * group, all = p.n_rows * group;
    const bool wide = kv_dpad(p.d) > 128;
    auto tiles = [&](long long t) {  // of t rows, that all sequences have together, at most
        const long long x = (all + p.n_seqs * (t - 1)) / t, y = p.n_seqs * ((rows + t - 1) / t);
        return x < y ? x : y;
    };
    auto seen = [&](long long t) {  // blocks that a tile of t rows sees, at most
        const long long in = (p.max_len + KV_BLOCK - 1) / KV_BLOCK, w = (window + (t + group - 1) / group + 2 * (KV_BLOCK - 1)) / KV_BLOCK;
        return (int)(window && w < in ? w : in);
    };
    // The step kernel takes what it has registers for, and more rows where the cache's blocks and the row tiles are few: it reads and
    // converts a block once for every 32 rows, but starts and ends in a third of the time.  By it and by the kernel for many rows: eight
    // times 5 tokens of 48 heads that share keys over 1 000 to 9 000 positions 27 us and 42; 7 tokens, all over 9 000, 38 and 41; 500 rows
    // of 32 heads over themselves 17 and 23, 700 26 and 27, 1 000 33 and 30, 2 048 83 and 59; 4 times 64 of 32 over 2 900 41 and 42.  The
    // border is where they meet for heads of 64 to 128; of wider ones some calls would be faster by the other (400 rows of 32 heads of 256
    // 40 and 34, 500 54 and 42), others not (700 of 16 47 and 52, 1 500 of 8 60 and 70).
    const long long few = tiles(KV_STEP_ROWS) * p.heads;
    int blocks = seen(KV_STEP_ROWS);
    const int chip = wide ? 256 : 512;  // workgroups of the step kernel at a time: registers for one to a compute unit, or two
    // It is launched with the most tiles that a sequence has for every one, and those that are not there cost their start: as much as is
    // saved at about 8 000 (64 sequences of 300 positions, 8 heads, one of 500 rows and the others of one: 38 us against 40 by the
    // kernel for many rows; of 700: 47 against 40; 256 sequences, one of 2 048 rows that see 128 positions: 205 against 35).
    const long long launched = p.n_seqs * ((rows + KV_STEP_ROWS - 1) / KV_STEP_ROWS) * p.heads;
    // More than two rounds of it, where tiles of 128 rows are half as many or fewer: their starts are what short windows and sequences have
    // (12 times 100 rows of 24 heads that see 100 positions 36 us, 24 by the other; 1 900 of 32 heads of 80 that see 100 35 and 23; 10
    // times 200 rows of 40 heads over themselves 54 and 38; 7 times about 240 of 16/2 heads of 256 93 and 44).
    const bool rounds = few > 2 * chip && few >= 2 * tiles(128) * p.heads;
    if (rows <= KV_STEP_ROWS || (few * (blocks > 1 ? blocks : 1) <= 24576 && launched - few <= 8192 && !rounds)) {
        // One workgroup to a compute unit: two to each read no faster and have more to join (one row over 4 000 positions of 32 heads
        // in 8 parts 11.8 us, in 16 13.4; 40 over 16 000 of 8 in 16 parts 19.3, in 32 22.8).  Sequences may differ in length, so
        // that parts of some end early: there, as many as the chip holds (the eight above in 4 parts 33 us, in 7 25; of wide heads no more
        // than one either: 8 times 6 tokens of 16/2 heads of 256 over 4 000 in 8 parts 29 us, in 16 44; 2 times 33 of 16 over 3 000 39 and 60).
        r.tile = KV_STEP_ROWS, r.tiles = (int)((rows + KV_STEP_ROWS - 1) / KV_STEP_ROWS);
        const long long want = (p.n_seqs > 1 ? chip : 256) / few, most = (blocks + 7) / 8;
        r.splits = (int)(want < most ? want : most);
        r.ragged = 2 * launched >= 3 * few;
    } else {
        // 256 rows convert a block half as often as two times 128, but are one workgroup to a compute unit, whose start and end nothing
        // covers (2 048 positions: 70 us against 61; 8 192: 787 against 820)
        r.tile = seen(128) >= 128 && rows > 128 && !wide ? 256 : 128;
        blocks = seen(r.tile);
        r.tiles = (int)tiles(r.tile);
        // Blocks that a compute unit goes through one after the other where n workgroups share `room` places: those of the longest; on
        // average; and in so many rounds, of the shortest, since behind a long past a second round is as long as the first.
        auto in_turn = [&](int n, int room, int longest) {
            const int end = (p.max_len + KV_BLOCK - 1) / KV_BLOCK, mean = end - p.max_rows / (2 * KV_BLOCK), shortest = end - p.max_rows / KV_BLOCK;
            auto one = [&](int x) { return (float)(x < longest ? x : longest); };
            return fmaxf((float)longest, fmaxf(n * one(mean) / room, (n + room - 1) / room * one(shortest)));
        };
        // Parts, one round of the chip at most: a workgroup's blocks one after the other (0.75 us each, 1.05 with two waves to a SIMD)
        // against what the join reads and writes (1 024 rows of 32 heads over themselves in one part 29 us, in two 41; behind 20 011
        // others 690 in one by that, 337 in two).
        const int units = r.tiles * p.heads, room = r.tile == 256 ? 256 : 512, want = room / units, most = (blocks + 7) / 8;
        const float join = (float)p.n_rows * heads_q * p.d * (8 / 4.5e6f);
        float least = (r.tile == 256 || units > 256 ? 1.05f : 0.75f) * in_turn(units, room, blocks);
        r.splits = 1;
        for (int x = 2; x <= want && x <= most; x++) {
            const float t = (r.tile == 256 || units * x > 256 ? 1.05f : 0.75f) * blocks / x + 5 + x * join;
            if (t < least) least = t, r.splits = x;
        }
        // Two halves of a workgroup to a tile, each with half of its blocks: where tiles are few, the last ones, which see most, are the
        // time.  One such workgroup to a compute unit, so at most two rounds, of which the second starts when the first's short
        // ones end (rows over themselves, in halves and not: 4 096 of 8 heads 72 us and 77, of 16 97 and 116, 8 192 of 8 170 and 216, but
        // 2 048 of 32 65 and 60).  Where there are no short ones, behind a long past, two rounds are worth it only against two of the
        // others (1 024 rows of 40 heads over 6 000: 190 us, 160 in tiles of 256; 20 times 96 rows of 32/8 heads over 6 000: 239 and 330).
        const int pairs = (int)tiles(128) * p.heads;
        if (!wide && pairs <= 512 && 0.58f * in_turn(pairs, 256, seen(128)) + (pairs > 256 ? 35 : 5) < least)
            r = {128, (int)tiles(128), 1, true, false};
    }
    if (r.splits < 1) r.splits = 1;
    // One tile more than there are, where a wave does not look at all sequences together: its workgroups look past the last one, so that
    // a sequence that cannot be is found also where it has no tile of its own.
    if (r.tile != KV_STEP_ROWS && p.n_seqs > 64) r.tiles++;
    return r;
}

// Parts of sequences and heads, each with as many tiles as a sequence has at most
inline long long step_units(const Kv& p, const KvPlan& plan) { return (long long)p.heads * p.n_seqs * plan.splits; }

// Whether the step kernel's workgroups go by tile.  A part's tiles on one XCD leave XCDs without work where parts are few (500 rows of
// 48 heads that share one: one XCD had all of them, 111 us against 23), and where most tiles are not there, those that are would be so
// many workgroups apart that they might all be dealt to the same few compute units (64 sequences of 300 positions, one of 100 rows,
// the others of one, 8 heads: 45 us against 21).
inline bool step_by_tile(const Kv& p, const KvPlan& plan)
{
    const long long units = step_units(p, plan);
    return plan.ragged || 8 * ((units + 7) / 8 * 8 - units) >= units;
}

long long kv_attention_workgroups(const Kv& p, const KvPlan& plan)
{
    if (plan.tile != KV_STEP_ROWS) return (long long)plan.tiles * p.heads * plan.splits;
    const long long units = step_units(p, plan);
    return (step_by_tile(p, plan) ? units : (units + 7) / 8 * 8) * plan.tiles;
}

size_t kv_attention_ws(const KvPlan& plan, int n_rows, int heads_q, int d)
{
    return plan.splits > 1 ? (size_t)plan.splits * n_rows * heads_q * (4 * (size_t)d + 8) + 512 : 0;
}

hipError_t launch_kv_attention(const Kv& p, const KvAttend& c, const KvPlan& plan, void* ws, hipStream_t st)
{
    AttendArgs a;
    a.kv = p, a.q = (const _Float16*)c.q, a.out = (_Float16*)c.out, a.ld_q = c.ld_q, a.ld_out = c.ld_out, a.heads_q = c.heads_q;
    a.group = Div(c.heads_q / p.heads), a.heads = Div(p.heads), a.splits = Div(plan.splits), a.tiles = Div(plan.tiles < 1 ? 1 : plan.tiles);
    a.units = Div((int)step_units(p, plan)), a.by_tile = step_by_tile(p, plan);
    a.scale = c.scale * LOG2E, a.causal = c.causal, a.window = c.window;
    const size_t total = (size_t)p.n_rows * c.heads_q;
    a.stat = (float2*)ws, a.part = (float*)((char*)ws + ((plan.splits * total * 8 + 255) & ~(size_t)255));
    a.vec = p.d % 8 == 0 && ((((uintptr_t)c.q | (uintptr_t)c.out) & 15) | (c.ld_q & 7) | (c.ld_out & 7)) == 0;
    const int dp = kv_dpad(p.d);
    hipError_t e;
    auto pick = [&](auto w) {
        constexpr int DP = decltype(w)::value;
        return plan.tile == KV_STEP_ROWS ? launch_step<DP>(a, plan, st)
               : plan.tile == 256        ? launch_prompt<(DP > 128 ? 128 : DP), 8, 1>(a, plan.tiles, st)  // (never that for more)
               : plan.halves             ? launch_prompt<(DP > 128 ? 128 : DP), 4, 2>(a, plan.tiles, st)
                                         : launch_prompt<DP, 4, 1>(a, plan.tiles, st);
    };
    switch (dp) {
        case 32: e = pick(std::integral_constant<int, 32>()); break;
        case 64: e = pick(std::integral_constant<int, 64>()); break;
        case 96: e = pick(std::integral_constant<int, 96>()); break;
        case 128: e = pick(std::integral_constant<int, 128>()); break;
        case 160: e = pick(std::integral_constant<int, 160>()); break;
        case 192: e = pick(std::integral_constant<int, 192>()); break;
        case 224: e = pick(std::integral_constant<int, 224>()); break;
        default: e = pick(std::integral_constant<int, 256>()); break;
    }
    if (e != hipSuccess || plan.splits == 1) return e;
    const unsigned quads = (unsigned)((total * ((p.d + 3) / 4) + 255) / 256);
    if (plan.splits > 16)
        kv_join_kernel<<<(unsigned)total, 256, 0, st>>>(a);
    else if (plan.splits > 4)
        kv_join_few_kernel<16><<<quads, 256, 0, st>>>(a);
    else
        kv_join_few_kernel<4><<<quads, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace llmint8
