// The pages of a cache: who names which (table, lens, refs), and copies of whole pages.
//
// A cache's book is small (a table entry a page and sequence, a count a page) and these kernels are bound by the latency of
// dependent steps, so each does its work in as few launches as its dependences allow: free and fork a workgroup a
// sequence (counts by integer atomics, whose order changes nothing), reserve one workgroup that scans, compact one launch
// where pages and table entries are few, else two over the pages, beyond 32768 pages three.  Copies are bound by HBM.
#pragma once
#include "common.h"

namespace tlin {

struct BookArgs {
    int32_t *table, *lens, *refs;
    const int32_t *ids;          // free: sequences; fork: parents; reserve: rows wanted
    const int32_t *children;     // fork
    int32_t *moves, *count, *status;
    int32_t *scratch;
    int32_t n;
    int32_t S, M, P, lr;
    int32_t stride;              // of the table
    // compact
    const int32_t *table_in, *refs_in;
    int32_t nblocks, counted;    // blocks of pages, and whether pages_count_kernel has counted them
    int32_t alone;               // the plan's one workgroup applies it too
};

__device__ __forceinline__ bool names_page(int id, int P) { return id >= 0 && id < P; }
// pages of a sequence of len rows
__device__ __forceinline__ int pages_of(int64_t len, int lr) { return (int)((len + (1 << lr) - 1) >> lr); }

// ---- free: one workgroup per listed sequence
__global__ __launch_bounds__(256) void pages_free_kernel(const BookArgs a)
{
    const int i = blockIdx.x, s = a.ids[i];
    if (s < 0 || s >= a.S) return;
    // the first that lists a sequence frees it
    int again = 0;
    for (int j = threadIdx.x; j < i; j += 256) again |= a.ids[j] == s;
    if (__syncthreads_or(again)) return;
    int32_t *row = a.table + (int64_t)s * a.stride;
    for (int j = threadIdx.x; j < a.M; j += 256) {
        const int id = row[j];
        if (names_page(id, a.P)) atomicSub(a.refs + id, 1);
        if (id != -1) row[j] = -1;
    }
    if (threadIdx.x == 0) a.lens[s] = 0;
}

// ---- fork: one workgroup per pair
__global__ __launch_bounds__(256) void pages_fork_kernel(const BookArgs a)
{
    const int i = blockIdx.x, from = a.ids[i], to = a.children[i];
    bool bad = from < 0 || from >= a.S || to < 0 || to >= a.S;
    int used = 0;
    if (!bad)
        for (int j = threadIdx.x; j < a.n; j += 256) used |= a.ids[j] == to || (j < i && a.children[j] == to);
    bad = __syncthreads_or(used) || bad;
    // (only this workgroup writes the child's length, and no workgroup the parent's: no pair names it as a child)
    if (!bad && a.lens[to] != 0) bad = true;
    __syncthreads();
    if (threadIdx.x == 0) a.status[i] = bad;
    if (bad) return;
    // a parent that some pair names as a child is passed over there; its rows are whole here
    const int len = min(max(a.lens[from], 0), a.M << a.lr);
    const int n = pages_of(len, a.lr);
    const int32_t *src = a.table + (int64_t)from * a.stride;
    int32_t *dst = a.table + (int64_t)to * a.stride;
    for (int j = threadIdx.x; j < a.M; j += 256) {
        int id = -1;
        if (j < n) {
            id = src[j];
            if (names_page(id, a.P)) atomicAdd(a.refs + id, 1);
        }
        dst[j] = id;
    }
    if (threadIdx.x == 0) a.lens[to] = len;
}

// Sum over the lanes below this one in the workgroup of 1024, and over all.  red: 16 values of LDS.
template <typename T>
__device__ __forceinline__ T block_scan(T x, T &total, T *red)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T v = x;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const T y = __shfl_up(v, off);
        if (lane >= off) v += y;
    }
    __syncthreads();
    if (lane == 63) red[wave] = v;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        const T r = red[w];
        before += w < wave ? r : 0;
        all += r;
    }
    total = all;
    return before + v - x;
}

// ---- reserve: one workgroup.
// What sequence s needs: pages for its new rows, and one in the place of a shared last page that is not full.
struct Need { int have, pages, copy; bool bad; };
__device__ __forceinline__ Need need_of(const BookArgs &a, int s)
{
    Need n = {0, 0, 0, false};
    const int want = a.ids[s], len = a.lens[s];
    if (want == 0) return n;
    if (want < 0 || len < 0 || (int64_t)len + want > (int64_t)a.M << a.lr) {
        n.bad = true;
        return n;
    }
    n.have = pages_of(len, a.lr);
    n.pages = pages_of((int64_t)len + want, a.lr) - n.have;
    if (len & ((1 << a.lr) - 1)) {
        const int last = a.table[(int64_t)s * a.stride + n.have - 1];
        if (names_page(last, a.P) && a.refs[last] > 1) n.copy = 1;
    }
    n.pages += n.copy;
    return n;
}

// scratch: first[S] (pages handed out before s), nth_copy[S] (twice the copies before s, odd where s has one; -1: s gets
// nothing), fresh[P] (free pages in order)
__global__ __launch_bounds__(1024) void pages_reserve_kernel(const BookArgs a)
{
    __shared__ int64_t red[16];
    __shared__ int red32[16];
    int32_t *first = a.scratch, *nth_copy = first + a.S, *fresh = nth_copy + a.S;
    const int tid = threadIdx.x;

    // pages wanted before every sequence: 32-bit sums would do for the pages there are, not for those asked for
    int64_t asked = 0;
    Need mine = {0, 0, 0, false};        // where each thread has one sequence at most
    for (int s0 = 0; s0 < a.S; s0 += 1024) {
        const int s = s0 + tid;
        const Need n = s < a.S ? need_of(a, s) : Need{0, 0, 0, false};
        mine = n;
        int64_t all;
        const int64_t at = asked + block_scan<int64_t>(n.bad ? 0 : n.pages, all, red);
        if (s < a.S) first[s] = (int)min(at, (int64_t)a.P + 1);
        asked += all;
    }
    const int most = (int)min(asked, (int64_t)a.P);
    // the free pages, lowest first, as far as they are asked for
    int found = 0;
    for (int p0 = 0; p0 < a.P && found < most; p0 += 16 * 1024) {
        // sixteen pages a thread, in the order of threads
        unsigned bits = 0;
        const int p = p0 + 16 * tid;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (p + e < a.P && a.refs[p + e] <= 0) bits |= 1u << e;
        int all;
        int at = found + block_scan<int>(__popc(bits), all, red32);
        while (bits) {
            const int e = __ffs(bits) - 1;
            bits &= bits - 1;
            if (at < most) fresh[at] = p + e;
            ++at;
        }
        found += all;
    }
    const int avail = min(found, most);
    __syncthreads();

    // who gets its pages, and the copies in order
    int copies = 0;
    for (int s0 = 0; s0 < a.S; s0 += 1024) {
        const int s = s0 + tid;
        const Need n = a.S <= 1024 ? mine : s < a.S ? need_of(a, s) : Need{0, 0, 0, false};
        const bool ok = s < a.S && !n.bad && (n.pages == 0 || (int64_t)first[s] + n.pages <= avail);
        int all;
        const int at = copies + block_scan<int>(ok ? n.copy : 0, all, red32);
        if (s < a.S) {
            a.status[s] = !ok;
            nth_copy[s] = ok ? 2 * at + n.copy : -1;
        }
        copies += all;
    }
    for (int i = tid; i < a.S; i += 1024)
        if (i >= copies) a.moves[2 * i] = a.moves[2 * i + 1] = -1;
    if (tid == 0) a.count[0] = copies;
    __syncthreads();      // every need has been read before anything changes

    // a wave a sequence: its pages
    const int lane = tid & 63;
    for (int s = tid >> 6; s < a.S; s += 16) {
        if (nth_copy[s] < 0) continue;
        const int want = a.ids[s], len = a.lens[s];
        if (want == 0) continue;
        const int have = pages_of(len, a.lr), end = pages_of((int64_t)len + want, a.lr);
        int32_t *row = a.table + (int64_t)s * a.stride;
        const int copy = nth_copy[s] & 1, nth = nth_copy[s] >> 1;
        const int at = first[s];
        for (int j = lane; j < end - have + copy; j += 64) {
            const int id = fresh[at + j], e = have - copy + j;
            if (copy && j == 0) {
                const int old = row[e];
                atomicSub(a.refs + old, 1);
                a.moves[2 * nth] = old;
                a.moves[2 * nth + 1] = id;
            }
            row[e] = id;
            a.refs[id] = 1;
        }
        if (lane == 0) a.lens[s] = len + want;
    }
}

// ---- compact
constexpr int kPagesPerBlock = 4096;

// live pages of every block of pages
__global__ __launch_bounds__(1024) void pages_count_kernel(const BookArgs a)
{
    __shared__ int red[16];
    const int p = blockIdx.x * kPagesPerBlock + 4 * threadIdx.x;
    int n = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) n += p + e < a.P && a.refs_in[p + e] > 0;
    block_scan<int>(n, all, red);
    if (threadIdx.x == 0) a.scratch[blockIdx.x] = all;
}

// The table and the counts after the moves, and the entries of moves behind the last: entries i0, i0 + step, ...  Tables and
// counts may be written in place: an entry is read and written by one thread, a hole's count and that of the page that
// moves into it by the hole's.
__device__ __forceinline__ void apply_moves(const BookArgs &a, int64_t i0, int64_t step)
{
    const int32_t *rank = a.scratch + a.nblocks;
    const int L = a.scratch[a.nblocks + a.P], K = a.count[0];
    for (int64_t i = i0; i < (int64_t)a.S * a.M; i += step) {
        const int64_t s = i / a.M, at = s * a.stride + (i - s * a.M);
        int id = a.table_in[at];
        // (a page that a table names and whose count is 0 goes nowhere: the entry stays)
        if (id >= L && id < a.P && rank[id] >= 0) id = a.moves[2 * rank[id] + 1];
        a.table[at] = id;
    }
    for (int64_t i = i0; i < a.P; i += step) {
        const int id = (int)i, n = a.refs_in[id];
        if (id < L) {
            if (n > 0) a.refs[id] = n;
            else {
                const int from = a.moves[2 * rank[id]];
                const int m = a.refs_in[from];
                a.refs[id] = m;
                a.refs[from] = 0;
            }
        } else if (n <= 0) a.refs[id] = 0;
        if (id >= K && id < a.P / 2) a.moves[2 * id] = a.moves[2 * id + 1] = -1;
    }
}
__global__ __launch_bounds__(256) void pages_apply_kernel(const BookArgs a)
{
    apply_moves(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

// With L live pages in all, the hole below L of rank i (holes counted from the lowest) takes the live page whose
// rank among the live ones is L - 1 - i.  rank[page] (behind the block counts) keeps i for holes
// below L and pages that move, -1 for free pages from L on.
__global__ __launch_bounds__(1024) void pages_plan_kernel(const BookArgs a)
{
    __shared__ int red[16];
    const int tid = threadIdx.x, b = blockIdx.x;
    int before = 0, live = 0, all;
    if (a.counted) {
        for (int k = tid; k < a.nblocks; k += 1024) {
            const int c = a.scratch[k];
            before += k < b ? c : 0;
            live += c;
        }
    } else {
#pragma unroll 8
        for (int k = tid; k < a.P; k += 1024) {
            const int c = a.refs_in[k] > 0;
            before += k < b * kPagesPerBlock ? c : 0;
            live += c;
        }
    }
    block_scan<int>(before, all, red);
    const int base = all;
    block_scan<int>(live, all, red);
    const int L = all;

    const int p = b * kPagesPerBlock + 4 * tid;
    int is[4], n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        is[e] = p + e < a.P && a.refs_in[p + e] > 0;
        n += is[e];
    }
    int r = base + block_scan<int>(n, all, red);      // live pages before p
    int32_t *rank = a.scratch + a.nblocks;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int id = p + e;
        if (id < a.P) {
            if (is[e] && id >= L) {
                const int i = L - 1 - r;
                a.moves[2 * i] = id;
                rank[id] = i;
            } else if (!is[e] && id < L) {
                const int i = id - r;
                a.moves[2 * i + 1] = id;
                rank[id] = i;
            } else if (id >= L) {
                rank[id] = -1;
            }
            r += is[e];
            if (id == L - 1) a.count[0] = L - r;      // holes below L
        }
    }
    if (L == 0 && b == 0 && tid == 0) a.count[0] = 0;
    if (b == 0 && tid == 0) a.scratch[a.nblocks + a.P] = L;
    if (a.alone) {
        __syncthreads();         // (what this workgroup has written it sees)
        apply_moves(a, tid, 1024);
    }
}

// ---- copy
struct CopyArgs {
    char *cache[2];
    int64_t layer[2], page[2], head[2], row[2];    // strides in bytes
    const int32_t *moves, *count;
    int32_t max_moves, P;
    int32_t layers, HK, R;
    int32_t row_pieces;         // 16-byte pieces of a row
    int32_t caches;             // 1 or 2
    int32_t flat[2];            // a page is one run of bytes
    int64_t pieces;             // 16-byte pieces of a page
    int32_t parts;              // shares that a page is cut into
};

// Work items: (move, layer, cache, part of the page), dealt to the workgroups in turn.  A thread has four pieces in
// flight at a time.
__global__ __launch_bounds__(256) void pages_copy_kernel(const CopyArgs a)
{
    const int n = a.count ? min(max(a.count[0], 0), a.max_moves) : a.max_moves;
    const int64_t items = (int64_t)n * a.layers * a.caches * a.parts;
    const int64_t per = (a.pieces + a.parts - 1) / a.parts;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        int64_t r = it;
        const int part = r % a.parts;
        r /= a.parts;
        const int c = r % a.caches;
        r /= a.caches;
        const int layer = r % a.layers, m = (int)(r / a.layers);
        const int from = a.moves[2 * m], to = a.moves[2 * m + 1];
        if (from < 0 || from >= a.P || to < 0 || to >= a.P) continue;
        char *const base = a.cache[c] + layer * a.layer[c];
        const char *src = base + from * a.page[c];
        char *dst = base + to * a.page[c];
        const int64_t lo = part * per, hi = min(lo + per, a.pieces);
        // byte offset of piece i of a page
        auto at = [&](int64_t i) __attribute__((always_inline)) {
            if (a.flat[c]) return i * 16;
            const int64_t row = i / a.row_pieces;
            const int h = (int)(row / a.R);
            return h * a.head[c] + (row - (int64_t)h * a.R) * a.row[c] + (i - row * a.row_pieces) * 16;
        };
        for (int64_t i = lo + threadIdx.x; i < hi; i += 4 * 256) {
            u32x4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * 256 < hi) x[u] = __builtin_nontemporal_load((const u32x4 *)(src + at(i + u * 256)));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * 256 < hi) __builtin_nontemporal_store(x[u], (u32x4 *)(dst + at(i + u * 256)));
        }
    }
}

}  // namespace tlin
