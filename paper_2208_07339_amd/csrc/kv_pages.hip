// kv_fork, kv_reserve, kv_compact, kv_copy: which sequence holds which pages of the key/value cache (layout: kv.h), and the copies
// that follow from it.
//
// The state is the tables and, for each page, how many table entries name it.  What a call does to them does not hang on the order in
// which its threads run: counts are changed by integer additions, and pages are given out by rank (sequences in order, the lowest free
// pages first).
#include "kv_pages.h"

#include "wave.h"

namespace llmint8 {

namespace {

__device__ __forceinline__ void flag(int* status, int bit)
{
    if (status) atomicOr(status, bit);
}

// ---- fork ------------------------------------------------------------------------------------------------------------------

constexpr int FORK_THREADS = 256;

struct ForkArgs {
    int* refs;
    int n_pages;
    int *pages, *kv_len, *slots, *status;
    int n, stride;
    const int* parent;
    int grow, columns;  // columns of the tables to a workgroup
    int4* list;
    int* count;
};

// Workgroup 0: lengths, slots and the list of ring copies.  The others: `columns` columns of all tables each, which makes the exchange
// of rows one in place: a workgroup has read its columns before it writes them.  A row's pages change their counts by the row's
// children less one.  Latency: three dependent round trips (parents and entries; counts and entries written).  2.3 us for 4 tables of
// 21 entries, about what a kernel that does nothing takes, 4.5 for 128 of 79, 5.3 for 16 of 2 302.
__global__ void __launch_bounds__(FORK_THREADS) kv_fork_kernel(const ForkArgs a)
{
    extern __shared__ int lds[];
    const int tid = threadIdx.x, n = a.n;
    int* const par = lds;         // [n] the parent, -1: none
    int* const child = lds + n;   // [n] children
    int* const rest = lds + 2 * n;
    const bool meta = blockIdx.x == 0;
    const int col0 = ((int)blockIdx.x - 1) * a.columns;
    bool bad = false, bad_page = false;

    int* const first = rest;          // [n] the lowest child             (workgroup 0)
    int* const slot = rest + n;       // [n] slots before
    int* const len = rest + 2 * n;    // [n] lengths before
    int* const spare = rest + 3 * n;  // [n] slots of sequences without children
    for (int i = tid; i < n; i += FORK_THREADS) {
        child[i] = 0;
        if (meta) first[i] = n;
    }
    __syncthreads();
    for (int i = tid; i < n; i += FORK_THREADS) {
        int p = a.parent[i];
        if (p < -1 || p >= n) bad = true, p = -1;
        par[i] = p;
        if (p >= 0) {
            atomicAdd(&child[p], 1);
            if (meta) atomicMin(&first[p], i);
        }
        if (meta) slot[i] = a.slots[i], len[i] = a.kv_len[i];
    }
    if (!meta) {
        // tile [n][columns]
#pragma unroll 4
        for (int t = tid; t < n * a.columns; t += FORK_THREADS) {
            const int r = t / a.columns, c = col0 + t % a.columns;
            const int e = a.pages[(long long)r * a.stride + (c < a.stride ? c : a.stride - 1)];
            if (c < a.stride && e >= a.n_pages) bad_page = true;
            rest[t] = c < a.stride && (unsigned)e < (unsigned)a.n_pages ? e : -1;
        }
        __syncthreads();
        for (int t = tid; t < n * a.columns; t += FORK_THREADS) {
            const int r = t / a.columns, c = col0 + t % a.columns, p = par[r], e = rest[t], k = child[r];
            if (e >= 0 && k != 1) atomicAdd(&a.refs[e], k - 1);
            if (c < a.stride && p != r) a.pages[(long long)r * a.stride + c] = p >= 0 ? rest[p * a.columns + t % a.columns] : -1;
        }
        if (bad_page) flag(a.status, LLMINT8_KV_BAD_PAGE);
        return;
    }

    if (bad) flag(a.status, LLMINT8_KV_BAD_BATCH);
    __syncthreads();
    if (tid >= 64) return;
    // One wave from here: ranks by counting flags below a lane.
    const unsigned long long below = (1ull << tid) - 1;
    int spares = 0, extras = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + tid;
        const bool there = i < n;
        const int p = there ? par[i] : -1;
        const bool empty = there && child[i] == 0, extra = p >= 0 && first[p] != i;
        const unsigned long long em = __ballot(empty), ex = __ballot(extra);
        if (empty) spare[spares + __popcll(em & below)] = slot[i];
        spares += __popcll(em), extras += __popcll(ex);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int x = 0, dead = extras;  // spare slots given to children, to sequences that end
    bool bad_len = false;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + tid;
        const bool there = i < n;
        const int p = there ? par[i] : -1;
        const bool extra = p >= 0 && first[p] != i, ends = there && p < 0;
        const unsigned long long ex = __ballot(extra), de = __ballot(ends);
        if (there) {
            const int k = extra ? x + __popcll(ex & below) : dead + __popcll(de & below);
            const int s = extra || ends ? spare[k] : slot[p];
            const int l = p >= 0 ? len[p] : 0;
            const bool ok = l >= 0 && l <= KV_MAX_LEN / 4;
            if (!ok) bad_len = true;
            if (extra) {
                const int from = l / KV_BLOCK > 1 ? (l / KV_BLOCK - 1) * KV_BLOCK : 0;
                a.list[k] = ok ? int4{slot[p], s, from, l - from} : int4{slot[p], s, 0, 0};
            }
            a.slots[i] = s;
            a.kv_len[i] = ok && l > 0 ? l + a.grow : l;
        }
        x += __popcll(ex), dead += __popcll(de);
    }
    if (tid == 0) a.count[0] = 0, a.count[1] = extras;
    if (bad_len) flag(a.status, LLMINT8_KV_BAD_BATCH);
}

// ---- a set of pages in LDS ---------------------------------------------------------------------------------------------------

constexpr int WIDE = 1024;  // threads of the kernels that go by such a set

// Sum of v over the threads before this one, and over all.  TURN: calls one behind the other have 0 and 1 in turn, so that one barrier
// is enough: what a call writes was read before the barrier of the one before it.
template <int TURN>
__device__ __forceinline__ int block_rank(int v, int& total)
{
    __shared__ int sums[2][WIDE / 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int incl = wave_upto(v, 0, [](int a, int b) { return a + b; });
    if (lane == 63) sums[TURN][w] = incl;
    __syncthreads();
    const int mine = lane < WIDE / 64 ? sums[TURN][lane] : 0;
    const int upto = wave_upto(mine, 0, [](int a, int b) { return a + b; });
    total = lane_of(upto, 63);
    return lane_of(upto - mine, __builtin_amdgcn_readfirstlane(w)) + incl - v;
}

// Pages as bits, with the number of set ones before each 256.
struct PageSet {
    unsigned long long* bits;  // [words] page p: bit p % 64 of word p / 64
    int* before;               // [groups]
    int groups, total;
    static constexpr int BATCH = 10;  // up to 10 240 pages in one

    static __host__ __device__ int groups_of(int n_pages) { return (n_pages + 255) / 256; }
    static __host__ size_t bytes(int n_pages) { return (size_t)groups_of(n_pages) * (4 * 8 + 4); }

    // The counts of a batch of words, a word to a wave instruction.
    struct Batch {
        int v[BATCH];
        __device__ __forceinline__ void load(const int* refs, int n_pages, int q0)
        {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int u = 0; u < BATCH; u++) {
                const int p = 64 * (q0 + u * (WIDE / 64)) + lane;
                v[u] = refs[p < n_pages ? p : n_pages - 1];
            }
        }
    };
    // The pages whose count says so.  batch: the first batch's counts (of words w, w + WIDE / 64, ..., for wave w).  Has a turn of
    // block_rank, TURN.
    template <int TURN, class F>
    __device__ __forceinline__ void make(char* at, const int* refs, int n_pages, Batch& batch, F f)
    {
        groups = groups_of(n_pages);
        bits = (unsigned long long*)at, before = (int*)(at + (size_t)groups * 32);
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = WIDE / 64;
        for (int q0 = w; q0 < 4 * groups; q0 += BATCH * waves) {
            if (q0 >= BATCH * waves) batch.load(refs, n_pages, q0);
#pragma unroll
            for (int u = 0; u < BATCH; u++) {
                const int q = q0 + u * waves;
                const unsigned long long m = __ballot(64 * q + lane < n_pages && f(batch.v[u]));
                if (lane == 0 && q < 4 * groups) bits[q] = m;
            }
        }
        __syncthreads();
        const int g = threadIdx.x;  // groups <= WIDE
        int c = 0;
        if (g < groups)
#pragma unroll
            for (int u = 0; u < 4; u++) c += __popcll(bits[4 * g + u]);
        const int r = block_rank<TURN>(c, total);
        if (g < groups) before[g] = r;
        __syncthreads();
    }
    // how many set ones there are before page p
    __device__ int rank(int p) const
    {
        int r = before[p >> 8];
        for (int q = p >> 8 << 2; q < p >> 6; q++) r += __popcll(bits[q]);
        return r + __popcll(bits[p >> 6] & ((1ull << (p & 63)) - 1));
    }
    // the k-th page (from 0) that is set, or with SET false that is not; there is such a one
    template <bool SET>
    __device__ int find(int k) const
    {
        int lo = 0, hi = groups;
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1, c = SET ? before[m] : 256 * m - before[m];
            if (c <= k)
                lo = m;
            else
                hi = m;
        }
        k -= SET ? before[lo] : 256 * lo - before[lo];
        int q = 4 * lo;
        unsigned long long m = SET ? bits[q] : ~bits[q];
        for (int u = 1; u < 4 && k >= __popcll(m); u++) {
            k -= __popcll(m);
            q++;
            m = SET ? bits[q] : ~bits[q];
        }
        int at = 0;
#pragma unroll
        for (int w = 32; w; w >>= 1) {
            const int c = __popcll((m >> at) & ((1ull << w) - 1));
            if (k >= c) k -= c, at += w;
        }
        return 64 * q + at;
    }
};

static_assert((LLMINT8_KV_MAX_PAGES + 255) / 256 <= WIDE, "a thread to a group");

// ---- reserve -----------------------------------------------------------------------------------------------------------------

constexpr int GIVEN = 2048;  // pages given out by one call that are listed first; where there are more, each is looked for by itself

struct ReserveArgs {
    int* refs;
    int n_pages;
    int* pages;
    const int *kv_len, *row_start;
    int *ready, *status;
    int n, stride;
    Div page;  // positions to a page
    int4* list;
    int* count;
    int more;
};

// A sequence's new positions old .. len - 1, in pages first .. end - 1 of its table.  false: they cannot be.
struct NewRows {
    int old, len, first, end;
};
__device__ __forceinline__ bool new_rows(const ReserveArgs& a, int b, NewRows& s)
{
    const long long n = (long long)a.row_start[b + 1] - a.row_start[b];
    const int len = a.kv_len[b];
    s = {};
    if (n < 0 || len < 0 || len > KV_MAX_LEN / 4) return false;
    s.old = s.len = len;
    if (n == 0 || len == 0) return true;
    const int end = a.page.quot(len - 1) + 1;
    if (n > len || end > a.stride) {
        s.old = s.len = 0;
        return false;
    }
    s.old = len - (int)n, s.first = a.page.quot(s.old), s.end = end;
    return true;
}

// One workgroup: a thread to two sequences and their first page each, which is all that single tokens have; then the pages behind those.
// A page is missing, or is to be replaced, or stays: that is settled for all before anything is changed, so that counts are those of
// the call's start.  Needs are ranked (sequences in order, a sequence's pages in order) and the r-th gets the r-th free page, which a
// set of the free pages in LDS finds.
// Latency: rows and lengths, entries, counts, the free pages' counts: four round trips, and the barriers of four rankings.  4.2 us for 128
// sequences (1 279 pages) of which none needs any, 9.5 where they all get a page of their own (943 pages), 11 for 940 pages of 20 prompts
// (9 405 pages).  Where a call gives thousands, by one workgroup's instructions: 14 for 2 048 pages of 4 prompts, 75 for 20 480 of 20.
__global__ void __launch_bounds__(WIDE) kv_reserve_kernel(const ReserveArgs a)
{
    extern __shared__ __align__(16) char mem[];
    const int tid = threadIdx.x, n = a.n, n4 = (n + 3) & ~3, per = (int)a.page.d / KV_BLOCK;
    int* const same = (int*)mem;     // [n4] a sequence's first page that others hold, too, and that it is to write; then its place among needs
    int* const need = same + n4;     // [n4] pages that it needs
    int* const behind = need + n4;   // [n4] pages behind the first, of the sequences before
    int* const second = behind + n4; // [n4] the first of those
    int* const given = second + n4;  // [GIVEN] the pages that are given out, in order
    char* const set = (char*)(given + GIVEN);
    // Counts for the set of free pages, ahead of what they wait for: where sequences are few, mostly nothing is needed, and they are left
    // until it is.
    PageSet::Batch batch;

    int entry[2], kept[2];
    NewRows s[2];
    bool ok[2], missing[2], shared[2], copy[2];
    int held[2], bad_page = 0;
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int b = 2 * tid + u;
        ok[u] = new_rows(a, b < n ? b : n - 1, s[u]);
        if (b >= n) s[u] = {}, ok[u] = true;
    }
    const bool ahead = n >= 32;
    if (ahead) batch.load(a.refs, a.n_pages, tid >> 6);
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int b = 2 * tid + u;
        const int e = a.pages[(long long)(b < n ? b : n - 1) * a.stride + s[u].first];
        const bool due = s[u].end > s[u].first;
        if (due && e >= a.n_pages) bad_page = 1;
        missing[u] = due && (unsigned)e >= (unsigned)a.n_pages;
        entry[u] = (unsigned)e < (unsigned)a.n_pages ? e : 0;
        held[u] = a.refs[entry[u]];
        shared[u] = due && !missing[u] && s[u].len / KV_BLOCK > s[u].old / KV_BLOCK && held[u] > 1;
        kept[u] = s[u].old / KV_BLOCK - s[u].first * per;
        if (b < n4) same[b] = shared[u] ? entry[u] : -1, second[b] = s[u].first + 1;
    }
    const int c0 = s[0].end > s[0].first ? s[0].end - s[0].first - 1 : 0, c1 = s[1].end > s[1].first ? s[1].end - s[1].first - 1 : 0;
    int T;  // pages behind the first ones
    const int r = block_rank<0>(c0 + c1, T);
    if (2 * tid < n4) behind[2 * tid] = r, behind[2 * tid + 1] = r + c0;
    // (block_rank's barrier: same[] is there)
    // How many want the page that a sequence shares, or -1 where a later one does: a wave to a sequence, its lanes to all of them.
    const int lane = tid & 63, w = tid >> 6;
    int x[4];
#pragma unroll
    for (int k = 0; k < 4; k++) x[k] = 64 * k + lane < n ? same[64 * k + lane] : -1;
    for (int b0 = w; b0 < n; b0 += WIDE) {
        const int p = b0 + WIDE / 64 * lane < n ? same[b0 + WIDE / 64 * lane] : -1;
        for (unsigned long long left = __ballot(p >= 0); left; left &= left - 1) {
            const int l = __ffsll(left) - 1, b = b0 + WIDE / 64 * l, page = lane_of(p, l);
            int all = 0;
            bool later = false;
            auto look = [&](int y, int q0) {
                const unsigned long long same_page = __ballot(y == page);
                all += __popcll(same_page);
                const int d = b - q0;  // those behind place d
                later |= d < 0 ? same_page != 0 : d < 63 && same_page >> (d + 1) != 0;
            };
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (64 * k < n) look(x[k], 64 * k);
            for (int q0 = 256; q0 < n; q0 += 64) look(q0 + lane < n ? same[q0 + lane] : -1, q0);
            if (lane == 0) need[b] = later ? -1 : all;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int b = 2 * tid + u;
        copy[u] = shared[u] && need[b] < held[u];
        if (b < n4) need[b] = missing[u] || copy[u];
    }
    __syncthreads();

    // The sequence that page t of those behind is of; its place in the tables.
    auto of = [&](int t) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1;
            if (behind[m] <= t)
                lo = m;
            else
                hi = m;
        }
        return lo;
    };
    auto column = [&](int b, int t) { return second[b] + t - behind[b]; };
    // Those to be replaced are marked in the table, by MARK + page; the others that are needed are what they were, no page of the pool (but for
    // those that look like marks): a sequence that is not served keeps its table.
    constexpr int MARK = -2147483647 - 1;
    auto marked = [&](int e) { return e < MARK + a.n_pages; };
    for (int t = tid; t < T; t += WIDE) {
        const int b = of(t), j = column(b, t);
        int* const at = a.pages + (long long)b * a.stride + j;
        const int e = *at;
        if ((unsigned)e < (unsigned)a.n_pages) {
            if ((long long)j * per >= a.kv_len[b] / KV_BLOCK || a.refs[e] <= 1) continue;
            *at = MARK + e;
        } else {
            if (e >= 0) bad_page = 1;
            if (marked(e)) *at = -1;
        }
        atomicAdd(&need[b], 1);
    }
    if (T) __syncthreads();

    const int n0 = 2 * tid < n4 ? need[2 * tid] : 0, n1 = 2 * tid < n4 ? need[2 * tid + 1] : 0;
    int N;
    const int rank = block_rank<1>(n0 + n1, N);
    bool late = false, served[2] = {true, true};
    int copies = 0;
    if (N) {
        PageSet free;
        if (!ahead) batch.load(a.refs, a.n_pages, tid >> 6);
        free.make<0>(set, a.refs, a.n_pages, batch, [](int c) { return c == 0; });
        const bool listed = N <= GIVEN;
        if (listed) {
            // a lane to a word, then a wave to each word that has some
            for (int q0 = w; q0 < 4 * free.groups; q0 += WIDE) {
                const int q = q0 + WIDE / 64 * lane;
                unsigned long long m = 0;
                int r = N;
                if (q < 4 * free.groups) {
                    m = free.bits[q];
                    r = free.before[q >> 2];
#pragma unroll
                    for (int y = 0; y < 3; y++) r += y < (q & 3) ? __popcll(free.bits[(q & ~3) + y]) : 0;
                }
                for (unsigned long long left = __ballot(m != 0 && r < N); left; left &= left - 1) {
                    const int l = __ffsll(left) - 1;
                    const unsigned long long ml = lane_of(m, l);
                    const int rl = lane_of(r, l) + __popcll(ml & ((1ull << lane) - 1));
                    if ((ml >> lane & 1) && rl < N) given[rl] = 64 * (q0 + WIDE / 64 * l) + lane;
                }
            }
            __syncthreads();
        }
        auto page_of = [&](int r) { return listed ? given[r] : free.find<true>(r); };
        served[0] = n0 == 0 || rank + n0 <= free.total, served[1] = n1 == 0 || rank + n0 + n1 <= free.total;
        if (N > free.total) {
            // A sequence that was to keep a page, since all others that hold it would get another, must not write to blocks of one that gets
            // none: then it is not served, either.  Those others are before it, and behind a sequence that is not served none gets a page, so
            // only what needs no page is left out here: no other sequence's pages change by it.  need[]: full blocks of those that go on
            // holding the page same[].  (Looked for by a thread each: calls that find the pool empty may take longer.)
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (2 * tid < n4) need[2 * tid + u] = copy[u] && !served[u] ? s[u].old / KV_BLOCK : -1;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (shared[u] && !copy[u])
                    for (int q = 0; q < 2 * tid + u; q++)
                        if (same[q] == entry[u] && need[q] > s[u].old / KV_BLOCK) served[u] = false;
            // (same[] is written to behind block_rank's barrier)
        }
        late = !served[0] || !served[1];
        int firsts = 0;
        const int f0 = missing[0] || copy[0], f1 = missing[1] || copy[1];
        if (T) {
            const int before = block_rank<1>(f0 + f1, firsts);
            if (2 * tid < n4) same[2 * tid] = served[0] ? before + f0 : -1, same[2 * tid + 1] = served[1] ? before + f0 + f1 : -1;
        }
        bool note[2];
#pragma unroll
        for (int u = 0; u < 2; u++) note[u] = copy[u] && served[u] && kept[u] > 0;
        const int k = block_rank<0>(note[0] + note[1], copies);
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int b = 2 * tid + u;
            if (!served[u] || !(missing[u] || copy[u])) continue;
            const int p = page_of(rank + (u ? n0 : 0));
            a.pages[(long long)b * a.stride + s[u].first] = p;
            a.refs[p] = 1;
            if (copy[u]) atomicSub(&a.refs[entry[u]], 1);
            if (note[u]) a.list[k + (u ? note[0] : 0)] = int4{entry[u], p, kept[u], 0};
        }
        for (int t0 = 0, base = 0; t0 < T; t0 += 2 * WIDE) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const int t = t0 + u * WIDE + tid;
                int* at = nullptr;
                int b = 0, e = 0;
                if (t < T) {
                    b = of(t);
                    at = a.pages + (long long)b * a.stride + column(b, t);
                    e = *at;
                }
                int all;
                const bool needed = (unsigned)e >= (unsigned)a.n_pages;
                const int q = base + (u ? block_rank<0>(needed, all) : block_rank<1>(needed, all));
                base += all;
                if (!needed) continue;
                const int firsts_before = same[b];
                if (firsts_before >= 0) {
                    const int p = page_of(q + firsts_before);
                    *at = p;
                    a.refs[p] = 1;
                    if (marked(e)) atomicSub(&a.refs[e - MARK], 1);
                } else if (marked(e)) {
                    *at = e - MARK;
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int b = 2 * tid + u;
        if (b >= n) continue;
        if (a.ready) a.ready[b] = ok[u] && served[u] ? s[u].len : 0;
        if (!ok[u]) flag(a.status, LLMINT8_KV_BAD_BATCH);
    }
    if (late) flag(a.status, LLMINT8_KV_NO_PAGE);
    if (bad_page) flag(a.status, LLMINT8_KV_BAD_PAGE);
    if (tid == 0) {
        a.count[0] = copies;
        if (!a.more) a.count[1] = 0;
    }
}

// ---- compact -----------------------------------------------------------------------------------------------------------------

// One workgroup: the list, and the counts moved along with it.  With U pages in use, the k-th of those from U on goes to the k-th free
// page below U; there are as many of both.  entries > 0: the tables, too, which saves a launch (4 us) where they are small.
// Latency, as above: 4.5 us with 48 tables of 42 entries and 1 589 pages, 8.7 with 25 005 pages.
__global__ void __launch_bounds__(WIDE) kv_compact_kernel(int* refs, int n_pages, int per, int* used_out, int4* list, int* count, int* pages, int entries)
{
    extern __shared__ __align__(16) char mem[];
    PageSet::Batch batch;
    batch.load(refs, n_pages, threadIdx.x >> 6);
    PageSet used;
    used.make<0>(mem, refs, n_pages, batch, [](int c) { return c != 0; });
    const int U = used.total, below = U < n_pages ? used.rank(U) : U;  // (used pages below U)
    for (int p = U + (int)threadIdx.x; p < n_pages; p += WIDE) {
        if (!(used.bits[p >> 6] >> (p & 63) & 1)) continue;
        const int k = used.rank(p) - below, to = used.find<false>(k);
        refs[to] = refs[p];
        refs[p] = 0;
        list[k] = int4{p, to, per, 0};
    }
    if (below < U)
        for (int i = threadIdx.x; i < entries; i += WIDE) {
            const int e = pages[i];
            if (e >= U && e < n_pages && (used.bits[e >> 6] >> (e & 63) & 1)) pages[i] = used.find<false>(used.rank(e) - below);
        }
    if (threadIdx.x == 0) {
        count[0] = U - below, count[1] = 0;
        if (used_out) *used_out = U;
    }
}

// Table entries that name a page of the list, which is in order of those, get its new number.
__global__ void __launch_bounds__(256) kv_rename_kernel(int* pages, long long entries, int n_pages, const int4* list, const int* count)
{
    const int n = count[0];
    if (n == 0) return;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= entries) return;
    const int e = pages[i];
    if (e < list[0].x || e >= n_pages) return;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (list[m].x <= e)
            lo = m;
        else
            hi = m;
    }
    const int4 v = list[lo];
    if (v.x == e) pages[i] = v.y;
}

// ---- copy ----------------------------------------------------------------------------------------------------------------------

struct CopyArgs {
    char *codes, *ring;
    unsigned* consts;
    int n_pages, n_slots, per, d;
    Div heads;
    const int4 *pages, *slots;
    const int* count;
    int max_pages, max_slots;
    int* status;
};

// n units of V from src to dst by the workgroup, four a thread in flight
template <class V>
__device__ __forceinline__ void move(V* __restrict__ dst, const V* __restrict__ src, int n)
{
    int i = threadIdx.x;
    for (; i + 768 < n; i += 1024) {
        V v[4];
#pragma unroll
        for (int u = 0; u < 4; u++) v[u] = src[i + 256 * u];
#pragma unroll
        for (int u = 0; u < 4; u++) dst[i + 256 * u] = v[u];
    }
    for (; i < n; i += 256) dst[i] = src[i];
}

// A workgroup to an entry and a head (of a ring also to keys or values), one after the other: how many there are only the device knows.
// V: what a row of the ring is moved in.  Bound by HBM: 133 MB read and written in two calls of 15.1 us each (4.4 TB/s), 130 MB in one of
// 26.6 (4.9 TB/s); a large copy by itself reaches 4.8 TB/s.
template <class V>
__global__ void __launch_bounds__(256) kv_copy_kernel(const CopyArgs a)
{
    const int heads = a.heads.d;
    int np = a.count[0], ns = a.count[1];
    np = np < 0 ? 0 : np > a.max_pages ? a.max_pages : np;
    ns = ns < 0 ? 0 : ns > a.max_slots ? a.max_slots : ns;
    const long long of_pages = (long long)np * heads, all = of_pages + 2ll * ns * heads;
    const int block = 2 * KV_BLOCK * kv_dpad(a.d);  // bytes
    for (long long x = blockIdx.x; x < all; x += gridDim.x) {
        if (x < of_pages) {
            const int k = a.heads.quot((int)x), g = (int)x - k * heads;
            const int4 m = a.pages[k];
            if ((unsigned)m.x >= (unsigned)a.n_pages || (unsigned)m.y >= (unsigned)a.n_pages || m.z < 0 || m.z > a.per) {
                if (threadIdx.x == 0) flag(a.status, LLMINT8_KV_BAD_PAGE);
                continue;
            }
            const long long from = ((long long)m.x * heads + g) * a.per, to = ((long long)m.y * heads + g) * a.per;
            move((u4*)(a.codes + to * block), (const u4*)(a.codes + from * block), m.z * (block / 16));
            move(a.consts + to, a.consts + from, m.z);
        } else {
            const int y = (int)(x - of_pages), k = a.heads.quot(y >> 1), g2 = y - 2 * k * heads;
            const int4 m = a.slots[k];
            if ((unsigned)m.x >= (unsigned)a.n_slots || (unsigned)m.y >= (unsigned)a.n_slots || m.z < 0 || m.w < 0 || m.w > KV_RING) {
                if (threadIdx.x == 0) flag(a.status, LLMINT8_KV_BAD_BATCH);
                continue;
            }
            const int row = a.d * 2 / (int)sizeof(V), p = m.z % KV_RING, n1 = p + m.w < KV_RING ? m.w : KV_RING - p;
            V* const ring = (V*)a.ring;
            const long long from = ((long long)m.x * 2 * heads + g2) * KV_RING * row, to = ((long long)m.y * 2 * heads + g2) * KV_RING * row;
            move(ring + to + (long long)p * row, ring + from + (long long)p * row, n1 * row);
            if (m.w > n1) move(ring + to, ring + from, (m.w - n1) * row);
        }
    }
}

}  // namespace

hipError_t launch_kv_fork(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, const int* parent, int grow,
                          const llmint8_kv_moves_t& m, hipStream_t st)
{
    // about 1 024 entries to a workgroup, at most 32 KiB of them
    int columns = 64;
    while (columns > 4 && columns * s.n_seqs > 1024) columns /= 2;
    const ForkArgs a = {p.refs, p.n_pages, s.pages, s.kv_len, s.slots, s.status, s.n_seqs, s.page_stride, parent, grow, columns, (int4*)m.slots, m.count};
    const int rest = columns > 4 ? columns : 4;  // (workgroup 0 has four words a sequence, too)
    kv_fork_kernel<<<1 + (s.page_stride + columns - 1) / columns, FORK_THREADS, (size_t)s.n_seqs * (2 + rest) * 4, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_reserve(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, const int* row_start, int* ready, int more,
                             const llmint8_kv_moves_t& m, hipStream_t st)
{
    const ReserveArgs a = {p.refs, p.n_pages, s.pages, s.kv_len, row_start, ready, s.status, s.n_seqs, s.page_stride, Div(p.page_tokens), (int4*)m.pages,
                           m.count, more};
    kv_reserve_kernel<<<1, WIDE, (size_t)((s.n_seqs + 3) & ~3) * 16 + GIVEN * 4 + PageSet::bytes(p.n_pages), st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, int* used, const llmint8_kv_moves_t& m, hipStream_t st)
{
    const long long entries = (long long)s.n_seqs * s.page_stride;
    const bool small = entries <= 8 * WIDE;
    kv_compact_kernel<<<1, WIDE, PageSet::bytes(p.n_pages), st>>>(p.refs, p.n_pages, p.page_tokens / KV_BLOCK, used, (int4*)m.pages, m.count, s.pages,
                                                                  small ? (int)entries : 0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || small) return e;
    kv_rename_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, st>>>(s.pages, entries, p.n_pages, (const int4*)m.pages, m.count);
    return hipGetLastError();
}

hipError_t launch_kv_copy(const llmint8_kv_cache_t& c, const llmint8_kv_moves_t& m, int* status, hipStream_t st)
{
    const CopyArgs a = {(char*)c.codes, (char*)c.ring, (unsigned*)c.consts, c.n_pages, c.n_slots, c.page_tokens / KV_BLOCK, c.d, Div(c.heads),
                        (const int4*)m.pages, (const int4*)m.slots, m.count, m.max_pages, m.max_slots, status};
    const long long most = ((long long)m.max_pages + 2ll * m.max_slots) * c.heads;
    const unsigned grid = (unsigned)(most < 2048 ? most : 2048);
    if (c.d % 8 == 0)
        kv_copy_kernel<u4><<<grid, 256, 0, st>>>(a);
    else
        kv_copy_kernel<unsigned short><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace llmint8
