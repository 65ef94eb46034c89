// The 8-bit key/value cache: its layout, and what its kernels share (kv_cache.hip, attention.hip).
//
// A page holds page_tokens positions of one sequence, a multiple of 32.  A block is 32 positions of one key/value head.  Blocks
// that are full are held as codes of absmax quantisation (Section 2.1) with one constant for the keys and one for the values;
// the positions behind the last full block are held as fp16 in a ring of 64 positions a sequence, which also still has the
// 32 positions before them.  So a code is made once, from fp16 values, whatever calls its block came in by, and a sequence
// that drops its last positions (at most 32) finds the fp16 values of the block it falls back into.
//
// Tiles.  Codes of a block are tiles of 32 positions x 32 features, 1 KiB, in the operand order of v_mfma_f32_32x32x16_f16,
// so that a wave loads an operand of two MFMAs with 16 bytes a lane and nothing has to be moved between lanes:
//   keys   (operand A of S^T = K Q^T): lane l holds position l % 32, features 16 (l / 32) .. + 15;
//   values (operand A of O^T = V^T P^T): lane l holds feature l % 32, positions 8 j + 4 (l / 32) + e, j, e = 0 .. 3, which are the
//          positions whose scores the MFMA left in this lane: P goes from accumulators to operand in place.
#pragma once
#include "../../include/llmint8.h"
#include "common.h"

namespace llmint8 {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr int KV_BLOCK = LLMINT8_KV_BLOCK;
constexpr int KV_RING = LLMINT8_KV_RING;
constexpr int KV_MAX_D = LLMINT8_KV_MAX_D;
constexpr int KV_MAX_LEN = 1 << 30;
__host__ __device__ inline int kv_dpad(int d) { return (d + 31) & ~31; }

// Division by a number that the host knows: m = (2^32 - 1) / d is not above 2^32 / d and less than 1 + 1 / d below it, so the product's high
// half is the quotient of n < 2^31 or one less.
struct Div {
    unsigned d, m;
    __host__ Div() = default;
    __host__ explicit Div(int x) : d((unsigned)x), m(0xffffffffu / (unsigned)x) {}
    __device__ __forceinline__ int quot(int n) const
    {
        const unsigned q = __umulhi((unsigned)n, m);
        return (int)(q + ((unsigned)n - q * d >= d));
    }
    __device__ __forceinline__ int rem(int n) const { return n - quot(n) * (int)d; }
};

// Cache and batch as the kernels take them.
struct Kv {
    int8_t* codes;           // [page][head][block][2][32 dpad]
    unsigned* consts;        // [page][head][block]: constant of the keys (fp16 bits, low half), of the values
    unsigned short* ring;    // [slot][head][2][64][d]
    const int* row_start;    // [n_seqs + 1]
    const int* kv_len;       // [n_seqs]
    const int* pages;        // [n_seqs][page_stride]
    const int* slots;        // [n_seqs], or NULL: the sequence's number
    int* status;             // or NULL
    int n_pages, n_slots, heads, d;
    Div bpp;  // blocks to a page
    int n_seqs, n_rows, page_stride, max_rows, max_len;
};

__device__ __forceinline__ void kv_flag(const Kv& p, int bit)
{
    if (p.status) atomicOr(p.status, bit);
}

// Rows and positions of a sequence.  Row i (0 .. n - 1) is at position len - n + i.
struct KvSeq {
    int row0, n, len, slot;
};

// false: what the arrays say of sequence b cannot be.  It then has no rows (rows out of order, or too many), or rows and no
// positions (the rest), so that what goes by these stays inside every array.
__device__ __forceinline__ bool kv_seq(const Kv& p, int b, KvSeq& s)
{
    s.row0 = p.row_start[b];
    const int row1 = p.row_start[b + 1];
    s.len = p.kv_len[b];
    s.slot = p.slots ? p.slots[b] : b;
    s.n = row1 - s.row0;
    const bool rows = s.row0 >= 0 && row1 >= s.row0 && row1 <= p.n_rows && s.n <= p.max_rows;
    const bool ok = rows && s.len >= 0 && s.len <= p.max_len && (long long)s.len <= (long long)p.page_stride * p.bpp.d * KV_BLOCK &&
                    (unsigned)s.slot < (unsigned)p.n_slots;
    if (!rows) s.row0 = 0, s.n = 0;
    if (!ok) s.len = 0, s.slot = 0;
    return ok;
}

// Unit x of those that the sequences have one after the other, count(s) each: its sequence and its number there.  The whole wave takes
// part, 64 sequences at a time.  false: there is no such unit.  wrong: a sequence looked at cannot be.
template <class F>
__device__ __forceinline__ bool kv_find(const Kv& p, int x, F count, int& b, KvSeq& s, int& i, bool& wrong)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += 64) {
        KvSeq t = {};
        int c = 0;
        if (b0 + lane < p.n_seqs) {
            if (!kv_seq(p, b0 + lane, t)) wrong = true;
            c = count(t);
        }
        int incl = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(incl, d);
            if (lane >= d) incl += y;
        }
        const unsigned long long past = __ballot(base + incl > x);
        if (past) {  // (the same for all lanes, and the compiler is to know it: what hangs on it stays scalar)
            const int l = __builtin_amdgcn_readfirstlane(__ffsll(past) - 1);
            b = b0 + l;
            i = __builtin_amdgcn_readfirstlane(x - base - __builtin_amdgcn_readlane(incl - c, l));
            s.row0 = __builtin_amdgcn_readlane(t.row0, l), s.n = __builtin_amdgcn_readlane(t.n, l);
            s.len = __builtin_amdgcn_readlane(t.len, l), s.slot = __builtin_amdgcn_readlane(t.slot, l);
            return true;
        }
        base += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// number of a block in codes and consts; -1: the table names no page
__device__ __forceinline__ long long kv_block(const Kv& p, int b, int head, int blk)
{
    const int at = p.bpp.quot(blk), page = p.pages[(long long)b * p.page_stride + at];
    if ((unsigned)page >= (unsigned)p.n_pages) return -1;
    return ((long long)page * p.heads + head) * p.bpp.d + (blk - at * (int)p.bpp.d);
}

__device__ __forceinline__ unsigned short* kv_ring_row(const Kv& p, int slot, int head, int kv, int pos)
{
    return p.ring + ((((long long)slot * p.heads + head) * 2 + kv) * KV_RING + (pos & (KV_RING - 1))) * p.d;
}

// LLMINT8_OK, or what is wrong with a cache and a batch
int kv_check(const llmint8_kv_cache_t* c, const llmint8_kv_batch_t* b);
Kv kv_args(const llmint8_kv_cache_t* c, const llmint8_kv_batch_t* b);

struct KvAppend {  // the rest of llmint8_kv_append's arguments
    const void *k, *v, *q;
    void* q_out;
    long long ld_k, ld_v, ld_q, ld_q_out;
    int heads_q;
    const float *cos, *sin;
    int n_pos, rot, pairs;
};
hipError_t launch_kv_append(const Kv& p, const KvAppend& c, hipStream_t st);
hipError_t launch_kv_read(const Kv& p, void* k_out, void* v_out, hipStream_t st);

struct KvAttend {  // the rest of llmint8_kv_attention's arguments
    const void* q;
    void* out;
    long long ld_q, ld_out;
    int heads_q;
    float scale;
    int causal, window;
};
// How a call's work is cut up: host arithmetic on the sizes alone.
struct KvPlan {
    int tile;    // rows (of all query heads that share keys) to a workgroup
    int tiles;   // tiles that a sequence has at most (tile = KV_STEP_ROWS), or that all have together
    int splits;  // parts of the positions, joined by a kernel of their own if more than one
    bool halves;  // (tile = 128) a tile's blocks on two halves of a workgroup
    bool ragged;  // (tile = KV_STEP_ROWS) most sequences have far fewer tiles than the one with the most
};
KvPlan kv_plan(const Kv& p, int heads_q, int window);  // window 0: none
size_t kv_attention_ws(const KvPlan& plan, int n_rows, int heads_q, int d);
long long kv_attention_workgroups(const Kv& p, const KvPlan& plan);  // without those of a join
hipError_t launch_kv_attention(const Kv& p, const KvAttend& a, const KvPlan& plan, void* ws, hipStream_t st);

}  // namespace llmint8
