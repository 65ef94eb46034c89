// kv_append and kv_read: what goes into the 8-bit key/value cache and what it holds (layout: kv.h).
//
// Both move data and compute next to nothing: bound by HBM, or by latency where a call brings one token a sequence.
#include "kv.h"

namespace llmint8 {

namespace {

// fp16 bits of a finite value: infinities become +-65504, NaN 0
__device__ __forceinline__ unsigned short finite(unsigned short x, bool& bad)
{
    if ((x & 0x7c00u) != 0x7c00u) return x;
    bad = true;
    return (x & 0x3ffu) ? (unsigned short)0 : (unsigned short)((x & 0x8000u) | 0x7bffu);
}

__device__ __forceinline__ us8 finite8(us8 v, bool& bad)
{
    // any exponent of all ones: rare, so the usual case costs a test of the whole
    bool any = false;
#pragma unroll
    for (int e = 0; e < 8; e++) any |= (v[e] & 0x7c00u) == 0x7c00u;
    if (any) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            unsigned short t = v[e];
            v[e] = finite(t, bad);
        }
    }
    return v;
}

// (a, b) turned: products and sums rounded one by one, so that the result does not hang on which of them a compiler fuses
__device__ __forceinline__ void turn(unsigned short& a, unsigned short& b, float c, float s)
{
#pragma clang fp contract(off)
    const float x = f16_bits_to_float(a), y = f16_bits_to_float(b);
    const float p = x * c, q = y * s, r = y * c, t = x * s;
    a = __builtin_bit_cast(unsigned short, (_Float16)(p - q));
    b = __builtin_bit_cast(unsigned short, (_Float16)(r + t));
}

struct Rotation {
    const float *cos, *sin;
    int n_pos, half;  // half: pairs to a head
    int pairs;
};

struct Rows {  // fp16 rows: row r, head g at p + r * ld + g * d
    const unsigned short* p;
    long long ld;
};

struct AppendArgs {
    Kv kv;
    Rows k, v, q;
    unsigned short* q_out;
    long long ld_q_out;
    int heads_q, q_group, head_groups;  // query heads to a workgroup; workgroups of key/value heads
    Rotation rot;
};

// Rows row .. row + n - 1 (positions pos ...) of heads h0 .. h1 - 1, rotated if turned, made finite if FINITE, to out(row number, head,
// feature, value): eight features at a time if VEC, which d, rot and everything's alignment then allow (halves of pairs lie in
// whole groups of 8), else one.  The work is that of threads 0 .. threads - 1; one has both halves of what it turns, so input and
// output may be the same.
template <bool VEC, bool FINITE, class Out>
__device__ __forceinline__ void move_rows(const Rows& in, const Rotation& rot, bool turned, int d, int row, int pos, int n, int h0, int h1,
                                          int thread, int threads, Out out, bool& bad)
{
    const int nh = h1 - h0, half = turned ? rot.half : 0;
    // what is turned, and the rest: loops of their own, so that a turn's requests go out together, whatever it moves.  (The next turn's
    // wait for it: its stores may be to what they read, for all that the compiler knows.)
    auto all = [&](int per, auto body) {
        const int total = n * nh * per;
#pragma unroll 4
        for (int t = thread; t < total; t += threads) {
            const int rest = t / per, u = t - rest * per, i = nh == 1 ? rest : rest / nh, gh = rest - i * nh;
            body(i, h0 + gh, u, in.p + (row + i) * in.ld + (long long)(h0 + gh) * d, (long long)(pos + i) * half);
        }
    };
    if constexpr (VEC) {
        if (half && !rot.pairs)
            all(half / 8, [&](int i, int g, int u, const unsigned short* src, long long at) {
                us8 a = *(const us8*)(src + 8 * u), b = *(const us8*)(src + half + 8 * u);
                const float *c = rot.cos + at + 8 * u, *s = rot.sin + at + 8 * u;
                const f4 cc[2] = {*(const f4*)c, *(const f4*)(c + 4)}, ss[2] = {*(const f4*)s, *(const f4*)(s + 4)};
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    unsigned short x = a[e], y = b[e];
                    turn(x, y, cc[e >> 2][e & 3], ss[e >> 2][e & 3]);
                    a[e] = x, b[e] = y;
                }
                if (FINITE) a = finite8(a, bad), b = finite8(b, bad);
                out(i, g, 8 * u, a);
                out(i, g, half + 8 * u, b);
            });
        if (half && rot.pairs)
            all(half / 4, [&](int i, int g, int u, const unsigned short* src, long long at) {
                us8 a = *(const us8*)(src + 8 * u);
                const f4 cc = *(const f4*)(rot.cos + at + 4 * u), ss = *(const f4*)(rot.sin + at + 4 * u);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    unsigned short x = a[2 * e], y = a[2 * e + 1];
                    turn(x, y, cc[e], ss[e]);
                    a[2 * e] = x, a[2 * e + 1] = y;
                }
                if (FINITE) a = finite8(a, bad);
                out(i, g, 8 * u, a);
            });
        if (d > 2 * half)
            all((d - 2 * half) / 8, [&](int i, int g, int u, const unsigned short* src, long long) {
                us8 a = *(const us8*)(src + 2 * half + 8 * u);
                if (FINITE) a = finite8(a, bad);
                out(i, g, 2 * half + 8 * u, a);
            });
    } else {
        if (half)
            all(half, [&](int i, int g, int u, const unsigned short* src, long long at) {
                const int ja = rot.pairs ? 2 * u : u, jb = rot.pairs ? 2 * u + 1 : u + half;
                unsigned short x = src[ja], y = src[jb];
                turn(x, y, rot.cos[at + u], rot.sin[at + u]);
                if (FINITE) x = finite(x, bad), y = finite(y, bad);
                out(i, g, ja, x);
                out(i, g, jb, y);
            });
        if (d > 2 * half)
            all(d - 2 * half, [&](int i, int g, int u, const unsigned short* src, long long) {
                unsigned short x = src[2 * half + u];
                if (FINITE) x = finite(x, bad);
                out(i, g, 2 * half + u, x);
            });
    }
}

__device__ __forceinline__ void put(unsigned short* p, us8 v) { *(us8*)p = v; }
__device__ __forceinline__ void put(unsigned short* p, unsigned short v) { *p = v; }
__device__ __forceinline__ unsigned larger(unsigned m, us8 v)
{
    const u4 y = __builtin_bit_cast(u4, v) & 0x7fff7fffu;
    return pk_max_u16(pk_max_u16(m, pk_max_u16(y[0], y[1])), pk_max_u16(y[2], y[3]));
}
__device__ __forceinline__ unsigned larger(unsigned m, unsigned short v) { return pk_max_u16(m, v & 0x7fffu); }

// One wave to a block that gets new tokens and a key/value head, HEADS waves to a workgroup (y < the heads' groups); the workgroups
// behind take such a block's tokens and q_group query heads each.  A block that gets full: keys, then values, go through LDS, where
// the codes are collected into tiles; their maximum is taken on the way.  The fp16 rows of the last two blocks go to the ring.
// Bound by HBM: 8 192 tokens of 40 heads of 128 with their queries read 252 MB and write 168 in 102 us, 4.1 TB/s (a copy: 4.76).
// Single tokens are latency: 96 sequences of 40 heads 15 us, of which blocks that get full are the longest.  (A workgroup to a block
// and head instead, its four waves meeting at barriers, took 134 and 18 us where this took 111 and 15, a wave to the keys and one to
// the values of a block and head 124 and 14.)
// A call that begins inside block f and ends more than a block later writes, for a later block c, the half of the ring that
// holds f's old rows: then the wave of f writes c's rows there, when it has read the old ones.
// LDS rows are 16 bytes longer than their data, so that the 16-byte reads of 32 rows at one feature spread over the banks.
constexpr int HEADS = 2;

// Between a wave's accesses to memory that its lanes share: they are done in order, and so they are to be compiled.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

template <bool VEC>
__global__ void __launch_bounds__(64 * HEADS) kv_append_kernel(const AppendArgs a)
{
    extern __shared__ __align__(16) unsigned short lds[];
    const Kv& p = a.kv;
    const int d = p.d, dpad = kv_dpad(d), LD = dpad + 8;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    int b, i;
    bool wrong = false;
    KvSeq s;
    auto blocks = [&](const KvSeq& t) {
        if (t.n == 0 || t.len == 0) return 0;
        if (t.len < t.n || (a.rot.half && t.len > a.rot.n_pos)) {
            wrong = true;
            return 0;
        }
        return (t.len - 1) / KV_BLOCK - (t.len - t.n) / KV_BLOCK + 1;
    };
    bool found;
    if (p.max_rows == 1) {  // one block a sequence: no need to count
        b = blockIdx.x, i = 0;
        if (!kv_seq(p, b, s)) wrong = true;
        found = blocks(s) > 0;
    } else {
        found = kv_find(p, blockIdx.x, blocks, b, s, i, wrong);
    }
    if (wrong) kv_flag(p, LLMINT8_KV_BAD_BATCH);
    if (!found) return;

    const int old = s.len - s.n, f = old / KV_BLOCK, e = s.len / KV_BLOCK, blk = f + i;
    const int lo = blk * KV_BLOCK, hi = lo + KV_BLOCK < s.len ? lo + KV_BLOCK : s.len;  // its positions that there are
    const int from = lo > old ? lo : old;                                               // the new ones: from .. hi - 1
    bool bad = false;

    if ((int)blockIdx.y >= a.head_groups) {
        const int h0 = ((int)blockIdx.y - a.head_groups) * a.q_group, h1 = h0 + a.q_group < a.heads_q ? h0 + a.q_group : a.heads_q;
        const int r0 = s.row0 + from - old;
        move_rows<VEC, false>(a.q, a.rot, a.rot.half > 0, d, r0, from, hi - from, h0, h1, threadIdx.x, 64 * HEADS,
                              [&](int r, int g, int j, auto v) { put(a.q_out + (r0 + r) * a.ld_q_out + (long long)g * d + j, v); }, bad);
        return;
    }
    const int head = blockIdx.y * HEADS + w;
    if (head >= p.heads) return;
    const bool full = hi - lo == KV_BLOCK;
    // the later block whose rows overwrite what this call reads of f
    const int clash = old % KV_BLOCK && f < e - 1 ? ((e - 1 - f) % 2 == 0 ? e - 1 : e) : -1;
    auto to_ring = [&](int block, int kv) {
        const int l = block * KV_BLOCK > old ? block * KV_BLOCK : old;
        const int n = (block + 1) * KV_BLOCK < s.len ? (block + 1) * KV_BLOCK - l : s.len - l;
        move_rows<VEC, true>(kv ? a.v : a.k, a.rot, kv == 0 && a.rot.half > 0, d, s.row0 + l - old, l, n, head, head + 1, lane, 64,
                             [&](int r, int, int j, auto v) { put(kv_ring_row(p, s.slot, head, kv, l + r) + j, v); }, bad);
    };
    if (!full) {
        if (blk != clash) to_ring(blk, 0), to_ring(blk, 1);
        if (bad) kv_flag(p, LLMINT8_KV_NOT_FINITE);
        return;
    }

    const long long at = kv_block(p, b, head, blk);
    const bool keep = blk >= e - 1 && blk != clash;  // to the ring, too
    unsigned short* const T = lds + w * KV_BLOCK * LD;
    if (dpad > d)
        for (int t = lane; t < KV_BLOCK * (dpad - d); t += 64) T[t / (dpad - d) * LD + d + t % (dpad - d)] = 0;
#pragma unroll
    for (int kv = 0; kv < 2; kv++) {
        unsigned m = 0;
        const int per = VEC ? d / 8 : d;
#pragma unroll 4
        for (int t = lane; t < (from - lo) * per; t += 64) {  // the rows that were there
            const int r = t / per, u = t - r * per;
            const unsigned short* src = kv_ring_row(p, s.slot, head, kv, lo + r);
            if constexpr (VEC) {
                const us8 v = *(const us8*)(src + 8 * u);
                m = larger(m, v);
                put(T + r * LD + 8 * u, v);
            } else {
                m = larger(m, src[u]);
                T[r * LD + u] = src[u];
            }
        }
        move_rows<VEC, true>(kv ? a.v : a.k, a.rot, kv == 0 && a.rot.half > 0, d, s.row0 + from - old, from, hi - from, head, head + 1, lane,
                             64, [&](int r, int, int j, auto v) {
                                 m = larger(m, v);
                                 put(T + (from - lo + r) * LD + j, v);
                                 if (keep) put(kv_ring_row(p, s.slot, head, kv, from + r) + j, v);
                             }, bad);
        wave_order();
        if (blk == f && clash >= 0) to_ring(clash, kv);
#pragma unroll
        for (int x = 32; x; x >>= 1) m = pk_max_u16(m, (unsigned)__shfl_xor((int)m, x));
        const unsigned c = (m & 0xffffu) > (m >> 16) ? m & 0xffffu : m >> 16;
        if (at >= 0) {
            if (lane == 0) ((unsigned short*)(p.consts + at))[kv] = (unsigned short)c;
            // codes: 16 bytes of a tile to a lane at a time
            const float fac = code_factor(f16_bits_to_float((unsigned short)c));
            int8_t* const dst = p.codes + at * (2ll * KV_BLOCK * dpad) + (long long)kv * KV_BLOCK * dpad;
            const int hh = lane >> 5, r = lane & 31;
            for (int g = 0; g < dpad / 32; g++) {
                unsigned o[4];
                if (kv == 0) {
                    const us8* src = (const us8*)(T + r * LD + 32 * g + 16 * hh);
                    const us8 x = src[0], y = src[1];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const us8& z = j < 2 ? x : y;
                        const int k = 4 * (j & 1);
                        o[j] = pack_low_bytes(code_bits(z[k], fac), code_bits(z[k + 1], fac), code_bits(z[k + 2], fac), code_bits(z[k + 3], fac));
                    }
                } else {
                    const unsigned short* src = T + 32 * g + r;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const unsigned short* z = src + (8 * j + 4 * hh) * LD;
                        o[j] = pack_low_bytes(code_bits(z[0], fac), code_bits(z[LD], fac), code_bits(z[2 * LD], fac), code_bits(z[3 * LD], fac));
                    }
                }
                *(u4*)(dst + (g * 64 + lane) * 16) = u4{o[0], o[1], o[2], o[3]};
            }
        }
        wave_order();
    }
    if (bad) kv_flag(p, LLMINT8_KV_NOT_FINITE);
    if (at < 0 && lane == 0) kv_flag(p, LLMINT8_KV_BAD_PAGE);
}

// c code / 127 for an integer n = c code that fp32 holds exactly: the correctly rounded fp32 quotient (reciprocal, and one
// correction by the exact remainder), then fp16.  An exact quotient that is no tie of two fp16 values is at least 2^-19 of
// itself away from one, so that the second rounding is that of the quotient.
__device__ __forceinline__ unsigned short value_bits(float n)
{
    const float r = 1.0f / 127.0f, q = n * r;
    return __builtin_bit_cast(unsigned short, (_Float16)__builtin_fmaf(__builtin_fmaf(-q, 127.0f, n), r, q));
}

// One workgroup to a block that holds some of the batch's rows, and a head: codes become fp16 rows in LDS and go out from there, whole
// rows at a time.  Bound by HBM, writes above all: 8 192 positions of 40 heads of 128 read 84 MB and write 168 in 54 us, 4.7 TB/s.
template <bool VEC>
__global__ void __launch_bounds__(256) kv_read_kernel(const Kv p, unsigned short* __restrict__ k_out, unsigned short* __restrict__ v_out)
{
    extern __shared__ __align__(16) unsigned short lds[];
    const int d = p.d, dpad = kv_dpad(d), LD = dpad + 8, tid = threadIdx.x, head = blockIdx.y;
    bool wrong = false;
    // Blocks of a sequence's rows, counted back from its last: the rows at positions before 0 are one more "block" each 32.
    auto blocks = [&](const KvSeq& t) {
        if (t.n == 0) return 0;
        const int first = t.len - t.n + (KV_MAX_LEN >> 1);  // above 0, the blocks' borders where they were
        return (first + t.n - 1) / KV_BLOCK - first / KV_BLOCK + 1;
    };
    int b, i;
    KvSeq s;
    const bool found = kv_find(p, blockIdx.x, blocks, b, s, i, wrong);
    if (wrong) kv_flag(p, LLMINT8_KV_BAD_BATCH);
    if (!found) return;
    const int old = s.len - s.n, f = (old + (KV_MAX_LEN >> 1)) / KV_BLOCK - (KV_MAX_LEN >> 1) / KV_BLOCK, blk = f + i;
    const int lo = blk * KV_BLOCK, hi = lo + KV_BLOCK < s.len ? lo + KV_BLOCK : s.len, from = lo > old ? lo : old;
    const long long row = s.row0 + (long long)(from - old);
    const int n = hi - from;
    const bool closed = blk >= 0 && blk < s.len / KV_BLOCK;
    long long at = -1;
    unsigned c = 0;
    if (closed) {
        at = kv_block(p, b, head, blk);
        if (at < 0) {
            if (tid == 0) kv_flag(p, LLMINT8_KV_BAD_PAGE);
        } else {
            c = p.consts[at];
        }
    }
    unsigned short* const outs[2] = {k_out, v_out};
#pragma unroll
    for (int kv = 0; kv < 2; kv++) {
        unsigned short* const out = outs[kv];
        if (!out) continue;
        if (at >= 0) {
            const int8_t* src = p.codes + at * (2ll * KV_BLOCK * dpad) + (long long)kv * KV_BLOCK * dpad;
            const float cf = f16_bits_to_float((unsigned short)(kv ? c >> 16 : c));
            __syncthreads();  // the keys' rows have been written out
            for (int t = tid; t < dpad * 2; t += 256) {
                const u4 x = *(const u4*)(src + 16 * t);
                const int g = t >> 6, hh = (t >> 5) & 1, r = t & 31;
                us8 y[2];
#pragma unroll
                for (int q = 0; q < 16; q++) y[q >> 3][q & 7] = value_bits((float)(int8_t)(x[q >> 2] >> (8 * (q & 3))) * cf);
                if (kv == 0) {
                    us8* dst = (us8*)(lds + r * LD + 32 * g + 16 * hh);
                    dst[0] = y[0], dst[1] = y[1];
                } else {
#pragma unroll
                    for (int q = 0; q < 16; q++) lds[(8 * (q >> 2) + 4 * hh + (q & 3)) * LD + 32 * g + r] = y[q >> 3][q & 7];
                }
            }
            __syncthreads();
        }
        const int per = VEC ? d / 8 : d;
        for (int t = tid; t < n * per; t += 256) {
            const int r = t / per, u = t % per, pos = from + r;
            unsigned short* dst = out + ((row + r) * p.heads + head) * d;
            const unsigned short* src = at >= 0 ? lds + (pos - lo) * LD : pos >= 0 ? kv_ring_row(p, s.slot, head, kv, pos) : nullptr;
            if (closed && at < 0) src = nullptr;
            if (VEC)
                *(us8*)(dst + 8 * u) = src ? *(const us8*)(src + 8 * u) : us8{};
            else
                dst[u] = src ? src[u] : (unsigned short)0;
        }
    }
}

}  // namespace

int kv_check(const llmint8_kv_cache_t* c, const llmint8_kv_batch_t* b)
{
    if (!c || !b || !c->codes || !c->consts || !c->ring || !b->row_start || !b->kv_len || !b->pages) return LLMINT8_INVALID_ARG;
    if (c->n_pages < 1 || c->page_tokens < 1 || c->n_slots < 1 || c->heads < 1 || c->d < 1) return LLMINT8_INVALID_ARG;
    if (b->n_seqs < 1 || b->n_rows < 1 || b->page_stride < 1 || b->max_rows < 1 || b->max_len < 0) return LLMINT8_INVALID_ARG;
    const uintptr_t words = (uintptr_t)b->row_start | (uintptr_t)b->kv_len | (uintptr_t)b->pages | (uintptr_t)b->slots | (uintptr_t)b->status;
    if (((uintptr_t)c->codes | (uintptr_t)c->consts | (uintptr_t)c->ring) & 15 || words & 3) return LLMINT8_INVALID_ARG;
    if (c->page_tokens % KV_BLOCK || c->page_tokens > KV_MAX_LEN || c->d > KV_MAX_D || c->heads > 65535 || b->max_len > KV_MAX_LEN / 4 ||
        b->n_rows > KV_MAX_LEN / 4 || b->n_seqs > (1 << 20))
        return LLMINT8_SHAPE;
    return LLMINT8_OK;
}

Kv kv_args(const llmint8_kv_cache_t* c, const llmint8_kv_batch_t* b)
{
    Kv p;
    p.codes = c->codes, p.consts = (unsigned*)c->consts, p.ring = (unsigned short*)c->ring;
    p.row_start = b->row_start, p.kv_len = b->kv_len, p.pages = b->pages, p.slots = b->slots, p.status = b->status;
    p.n_pages = c->n_pages, p.bpp = Div(c->page_tokens / KV_BLOCK), p.n_slots = c->n_slots, p.heads = c->heads, p.d = c->d;
    p.n_seqs = b->n_seqs, p.n_rows = b->n_rows, p.page_stride = b->page_stride;
    p.max_rows = b->max_rows < b->n_rows ? b->max_rows : b->n_rows, p.max_len = b->max_len;
    return p;
}

// Blocks that a call's rows lie in, at most: a sequence of n rows touches (n + 62) / 32.
inline long long most_blocks(const Kv& p)
{
    const long long a = ((long long)p.n_rows + 62ll * p.n_seqs) / KV_BLOCK, b = (long long)p.n_seqs * ((p.max_rows + 62) / KV_BLOCK);
    return a < b ? a : b;
}

inline size_t block_lds(int d) { return (size_t)KV_BLOCK * (kv_dpad(d) + 8) * 2; }

hipError_t launch_kv_append(const Kv& p, const KvAppend& c, hipStream_t st)
{
    AppendArgs a;
    a.kv = p;
    a.k = {(const unsigned short*)c.k, c.ld_k}, a.v = {(const unsigned short*)c.v, c.ld_v}, a.q = {(const unsigned short*)c.q, c.ld_q};
    a.q_out = (unsigned short*)c.q_out, a.ld_q_out = c.ld_q_out, a.heads_q = c.heads_q;
    a.rot = {c.cos, c.sin, c.n_pos, c.rot / 2, c.pairs};
    const bool has_q = c.q && !(c.q == c.q_out && c.rot == 0);
    auto aligned = [](const void* q, long long ld) { return ((uintptr_t)q & 15) == 0 && ld % 8 == 0; };
    bool vec = p.d % 8 == 0 && aligned(c.k, c.ld_k) && aligned(c.v, c.ld_v);
    if (has_q) vec = vec && aligned(c.q, c.ld_q) && aligned(c.q_out, c.ld_q_out);
    if (c.rot) vec = vec && aligned(c.cos, 0) && aligned(c.sin, 0) && c.rot % (c.pairs ? 8 : 16) == 0;
    const int rows = p.max_rows < KV_BLOCK ? p.max_rows : KV_BLOCK;
    // query heads to a workgroup: about four groups of 8 features to a thread, or 16 where there are more than enough workgroups (17 550
    // tokens of 48 heads 118 and 101 us; eight times five tokens of 48 heads 4.1 and 8).  Not with accesses of two bytes, whose turns
    // are eight times as many (8 192 tokens of 32 heads of 80, 20 features rotated: 102 us, and 124 with the larger groups).
    const int of4 = 512 / (rows * ((p.d + 7) / 8)), g4 = of4 < 1 ? 1 : of4;
    const int g = has_q && vec && most_blocks(p) * ((c.heads_q + g4 - 1) / g4) > 4096 ? 2048 / (rows * ((p.d + 7) / 8)) : g4;
    a.q_group = g < 1 ? 1 : has_q && g > c.heads_q ? c.heads_q : g;
    a.head_groups = (p.heads + HEADS - 1) / HEADS;
    const int qy = has_q ? (c.heads_q + a.q_group - 1) / a.q_group : 0;
    const dim3 grid((unsigned)most_blocks(p), a.head_groups + qy);
    if (vec)
        kv_append_kernel<true><<<grid, 64 * HEADS, HEADS * block_lds(p.d), st>>>(a);
    else
        kv_append_kernel<false><<<grid, 64 * HEADS, HEADS * block_lds(p.d), st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_read(const Kv& p, void* k_out, void* v_out, hipStream_t st)
{
    const dim3 grid((unsigned)most_blocks(p), p.heads);
    const bool vec = p.d % 8 == 0 && (((uintptr_t)k_out | (uintptr_t)v_out) & 15) == 0;
    if (vec)
        kv_read_kernel<true><<<grid, 256, block_lds(p.d), st>>>(p, (unsigned short*)k_out, (unsigned short*)v_out);
    else
        kv_read_kernel<false><<<grid, 256, block_lds(p.d), st>>>(p, (unsigned short*)k_out, (unsigned short*)v_out);
    return hipGetLastError();
}

}  // namespace llmint8
