// How the work of a paged attention call is cut: on the device, from the lengths that only it knows.
//
// An item is a (sequence, key head, query block): TB = BM / G new rows of a sequence with the G query heads that share
// the key head, BM rows for the matrix cores, over the rows of the cache that its last row sees.  All items laid end to
// end, each as long as the rows it reads, are cut into equal shares, one a workgroup: whatever the lengths are, every
// workgroup streams the same number of rows, a long sequence is spread over many, and short ones follow each other in one.
// An item that a cut goes through is finished by the merge kernel from partials (O, m, l) in the workspace; a
// workgroup has two slots for them, for the item that its share begins in the middle of and for the one that it ends in
// the middle of.  Every workgroup finds its share by itself (a scan over the sequences, 1 to 2 us) and leaves a
// record of the item that it ends in the middle of, which is all that the merge kernel has to know: nothing about a call is
// planned on the host or kept from one call to the next.
//
// With c rows before the new ones, block i reads u(i) = c + min(W, (i + 1) TB) rows (all of them alike without the causal
// mask), so the first n blocks of a head read n c + TB n (n + 1) / 2 rows, less what the last block lacks: every
// position is found without a list of items.
#pragma once
#include "common.h"

namespace tlin {

struct PagedArgs {
    const void *Q, *K, *V;
    const int32_t *table, *lens, *starts;
    void *O;
    float *lse;
    float *Opart, *Mpart, *Lpart;        // [2 shares][BM][DK], [2 shares][BM]
    struct CutItem *cuts;                // [shares]
    int64_t q_sh, q_sr, o_sh, o_sr;      // element strides
    int64_t k_sp, k_sh, k_sr, v_sp, v_sh, v_sr;
    int32_t S, T, HK, G;                 // G: query heads of a key head
    int32_t D;
    int32_t M, P, lr;                    // table width, pages, log2 of a page's rows
    int32_t table_stride;
    int32_t TB, BM;                      // new rows of a query block, rows of a workgroup
    int32_t shares;                      // workgroups that the work is cut for
    int32_t least;                       // rows of a share at least, a multiple of 64
    int32_t causal, out_bf16;
    float scale, c;                      // c = scale log2(e)
};

// The item that a share ends in the middle of: its partials are part 0 in slot 2 w + 1 of that share w, part k in slot
// 2 (w + k) of the k-th share after it.
struct CutItem {
    int32_t rows;            // (new row, query head) pairs; 0: the share ends with its last item, or a share holds all tiles
    int32_t row, head;       // first new row, first query head
    int32_t part0, part1;    // the parts that hold tiles: part0 .. part1 - 1
    int32_t pad[3];
};

// The kernel's arguments, to be read again from here on: what is used in one place of a long kernel does not
// have to stay in scalar registers through the rest of it (kept, they were spilled: up to 167 of them).
typedef const __attribute__((address_space(4))) PagedArgs ConstPagedArgs;
__device__ __forceinline__ ConstPagedArgs *args_again()
{
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return (ConstPagedArgs *)p;
}

// What starting an item costs (queries, first tiles, output), in rows of the cache: part of its length in the cuts.
constexpr int kItemRows = 64;

struct Sequence {
    int first, W, len;       // first new row, new rows, rows
    int nqb;                 // query blocks
    int before;              // rows that all of its blocks read (see above)
};

template <typename A>
__device__ __forceinline__ Sequence sequence_of(const A &a, int s)
{
    Sequence q;
    q.first = min(max(a.starts[s], 0), a.T);
    q.W = max(min(a.starts[s + 1], a.T) - q.first, 0);
    q.len = (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.M << a.lr);
    q.nqb = (q.W + a.TB - 1) / a.TB;
    // (a length below the number of new rows, which no caller means: the rows before the first see nothing)
    q.before = a.causal ? max(q.len - q.W, 0) : max(q.len, 1);
    return q;
}
// rows read by block i, and by the first n blocks of a head (n <= nqb), each with its start
template <typename A>
__device__ __forceinline__ int64_t block_rows(const A &a, const Sequence &q, int i)
{
    return kItemRows + (a.causal ? (int64_t)q.before + min((int64_t)q.W, (int64_t)(i + 1) * a.TB) : (int64_t)q.before);
}
template <typename A>
__device__ __forceinline__ int64_t rows_before(const A &a, const Sequence &q, int n)
{
    int64_t r = (int64_t)n * (q.before + kItemRows);
    if (a.causal) {
        r += (int64_t)a.TB * ((int64_t)n * (n + 1) / 2);
        if (n == q.nqb) r -= (int64_t)n * a.TB - q.W;
    }
    return r;
}
// key tiles of an item up to offset x of its length
template <int BN>
__device__ __forceinline__ int tiles_to(int64_t x) { return x <= kItemRows ? 0 : (int)((x - kItemRows + BN - 1) / BN); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Where a share begins, and how the shares are cut.
struct Place {
    int64_t total, quota;    // rows in all, rows of a share
    int s, head, qb;         // the item at the position asked for
    int64_t x;               // offset of the position inside that item
    Sequence q;
};

// red, off, s: of the search.  place, left: a wave's own place in its share while it works on an item (kept in scalar
// registers they were spilled).
struct PlaceLds { int64_t red[8]; int64_t off; int s; Place place[8]; int64_t left[8]; };

// The item at position w * quota, for a workgroup of NT threads (false: w is behind the last share).
template <int NT, typename A>
__device__ __forceinline__ bool find_place(const A &a, int w, Place &p, PlaceLds &lds)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int run = (a.S + NT - 1) / NT;       // sequences of a thread, next to each other
    const int lo = min(tid * run, a.S), hi = min(lo + run, a.S);
    int64_t sum = 0;
    for (int s = lo; s < hi; ++s) {
        const Sequence q = sequence_of(a, s);
        sum += a.HK * rows_before(a, q, q.nqb);
    }
    int64_t upto = sum;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const int64_t y = __shfl_up(upto, off);
        if (lane >= off) upto += y;
    }
    if (lane == 63) lds.red[wave] = upto;
    __syncthreads();
    int64_t total = 0, before = upto - sum;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) {
        before += k < wave ? lds.red[k] : 0;
        total += lds.red[k];
    }
    p.total = uniform(total);
    const int64_t even = (p.total + a.shares - 1) / a.shares;
    p.quota = uniform(even <= a.least ? (int64_t)a.least : (even + 63) / 64 * 64);
    const int64_t pos = w * p.quota;
    if (pos >= p.total) return false;
    if (pos >= before && pos < before + sum) {
        int64_t at = before;
        for (int s = lo; s < hi; ++s) {
            const Sequence q = sequence_of(a, s);
            const int64_t n = a.HK * rows_before(a, q, q.nqb);
            if (pos < at + n) {
                lds.s = s;
                lds.off = pos - at;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    p.s = uniform(lds.s);
    int64_t off = uniform(lds.off);
    Sequence q = sequence_of(a, p.s);
    q.first = uniform(q.first); q.W = uniform(q.W); q.len = uniform(q.len); q.nqb = uniform(q.nqb); q.before = uniform(q.before);
    p.q = q;
    const int64_t head = rows_before(a, q, q.nqb);
    p.head = uniform((int)(off / head));
    off -= p.head * head;
    int lo_b = 0, hi_b = q.nqb - 1;            // the last block that begins at or before off
    while (lo_b < hi_b) {
        const int mid = (lo_b + hi_b + 1) >> 1;
        if (rows_before(a, q, mid) <= off) lo_b = mid;
        else hi_b = mid - 1;
    }
    p.qb = uniform(lo_b);
    p.x = uniform(off - rows_before(a, q, p.qb));
    return true;
}

// The item after (s, head, qb); the caller knows that there is one.
template <typename A>
__device__ __forceinline__ void next_item(const A &a, Place &p)
{
    p.x = 0;
    if (++p.qb < p.q.nqb) return;
    p.qb = 0;
    if (++p.head < a.HK) return;
    p.head = 0;
    do {
        ++p.s;
        const Sequence q = sequence_of(a, p.s);
        p.q.first = uniform(q.first); p.q.W = uniform(q.W); p.q.len = uniform(q.len); p.q.nqb = uniform(q.nqb); p.q.before = uniform(q.before);
    } while (p.q.nqb == 0 && p.s + 1 < a.S);
}

// The items of share w, one after another: work(place, first tile, last tile, whole, slot) for each, and the record of
// the one that the share ends in the middle of.
template <int NT, int BN, typename F>
__device__ __forceinline__ void share_items(int w, PlaceLds &lds, F work)
{
    const int wave = uniform((int)threadIdx.x >> 6);
    ConstPagedArgs &a = *args_again();
    Place p;
    CutItem cut = {};
    const bool any = find_place<NT>(a, w, p, lds);
    if (any) {
        int64_t left = min(p.quota, p.total - w * p.quota);
        for (;;) {
            int64_t n;
            {
                ConstPagedArgs &b = *args_again();
                n = block_rows(b, p.q, p.qb);
            }
            const int64_t x1 = min(n, p.x + left);
            const int t0 = tiles_to<BN>(p.x), t1 = tiles_to<BN>(x1), nt = tiles_to<BN>(n);
            if (t0 < t1) {
                lds.place[wave] = p;
                lds.left[wave] = left;
                work(p, t0, t1, t0 == 0 && t1 == nt, 2 * w + (p.x > 0 ? 0 : 1));
                asm volatile("" ::: "memory");
                const Place &o = lds.place[wave];
                p.total = uniform(o.total); p.quota = uniform(o.quota);
                p.s = uniform(o.s); p.head = uniform(o.head); p.qb = uniform(o.qb); p.x = uniform(o.x);
                p.q.first = uniform(o.q.first); p.q.W = uniform(o.q.W); p.q.len = uniform(o.q.len);
                p.q.nqb = uniform(o.q.nqb); p.q.before = uniform(o.q.before);
                left = uniform(lds.left[wave]);
            }
            ConstPagedArgs &b = *args_again();
            const int64_t len = block_rows(b, p.q, p.qb), x = min(len, p.x + left);
            left -= x - p.x;
            if (left <= 0) {
                // the cut goes through an item that begins here
                if (x < len && p.x == 0) {
                    const int tiles = tiles_to<BN>(len), tile1 = tiles_to<BN>(x);
                    const int last = (int)((len - x + p.quota - 1) / p.quota);       // shares after this one with a part of it
                    // (a part is empty where it ends before the first tile, or begins behind the last)
                    const int part0 = tile1 == 0, part1 = tiles_to<BN>(x + (last - 1) * p.quota) < tiles ? last + 1 : last;
                    if (part1 - part0 > 1) {
                        cut.rows = min(b.TB, p.q.W - p.qb * b.TB) * b.G;
                        cut.row = p.q.first + p.qb * b.TB;
                        cut.head = p.head * b.G;
                        cut.part0 = part0;
                        cut.part1 = part1;
                    }
                }
                break;
            }
            next_item(b, p);
        }
    }
    if (threadIdx.x == 0) args_again()->cuts[w] = cut;
}

}  // namespace tlin
