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

// n / d for 0 <= n < 2^31 by a multiplication: m = ceil(2^k / d), k = 31 + ceil(log2 d), from the host.
struct Divide { uint32_t m; int32_t k; };
__device__ __forceinline__ int divide(int n, uint32_t m, int k) { return (int)((uint64_t)(uint32_t)n * m >> k); }

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
    Divide by_TB;
    int32_t shares;                      // workgroups that the work is cut for
    double per_share;                    // 1 / shares
    float per_G;                         // 1 / G: (r + 1/2) / G rounds down to r / G for the rows of a workgroup
    int32_t start;                       // what starting an item costs, in rows of the cache (even)
    int32_t causal, out_bf16;
    float scale, c;                      // c = scale log2(e)
};

// The item that a share ends in the middle of: its partials are part 0 in slot 2 w + 1 of that share w, part k in slot
// 2 (w + k) of the k-th share after it.
struct CutItem {
    int32_t rows;            // (new row, query head) pairs; 0: the share ends with its last item
    int32_t row, head;       // first new row, first query head
    int32_t parts;
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

// How far a row's logits may exceed its reference point, 8 base-2 units in units of the products.  A number for any scale: an
// infinite step (scales below 1.63e-38) would leave a reference of -infinity where it is.
__device__ __forceinline__ float reference_step(float c) { return fminf(8.0f / c, 3.402823466e38f); }

// Rows that a cut leaves of an item behind it at least.
constexpr int kShortest = 128;

struct Sequence {
    int first, W, len;       // first new row, new rows, rows
    int nqb;                 // query blocks
    int before;              // rows that all of its blocks read (see above)
};

// a / b for 0 <= a, 0 < b, a / b below 2^20: an approximate quotient is off by at most one
__device__ __forceinline__ int quotient(int64_t a, int64_t b)
{
    int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
    int64_t r = a - q * b;
    while (r < 0) { --q; r += b; }
    while (r >= b) { ++q; r -= b; }
    return q;
}

template <typename A>
__device__ __forceinline__ Sequence complete(const A &a, int first, int W, int len)
{
    Sequence q;
    q.first = first;
    q.W = W;
    q.len = len;
    q.nqb = divide(W + a.TB - 1, a.by_TB.m, a.by_TB.k);
    // (a length below the number of new rows, which no caller means: the rows before the first see nothing)
    q.before = a.causal ? max(len - W, 0) : max(len, 1);
    return q;
}
template <typename A>
__device__ __forceinline__ Sequence sequence_of(const A &a, int s)
{
    const int first = min(max(a.starts[s], 0), a.T);
    return complete(a, first, max(min(a.starts[s + 1], a.T) - first, 0), (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.M << a.lr));
}
// rows read by block i, and by the first n blocks of a head (n <= nqb)
template <typename A>
__device__ __forceinline__ int64_t block_rows(const A &a, const Sequence &q, int i)
{
    return a.causal ? (int64_t)q.before + min((int64_t)q.W, (int64_t)(i + 1) * a.TB) : (int64_t)q.before;
}
template <typename A>
__device__ __forceinline__ int64_t rows_before(const A &a, const Sequence &q, int n)
{
    int64_t r = (int64_t)n * q.before;
    if (a.causal) {
        r += (int64_t)a.TB * ((int64_t)n * (n + 1) / 2);
        if (n == q.nqb) r -= (int64_t)n * a.TB - q.W;
    }
    return r;
}
// key tiles of an item up to offset x of its length
template <int BN>
__device__ __forceinline__ int tiles_to(int64_t x, int start) { return x <= start ? 0 : (int)((x - start + BN - 1) / BN); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Where a share begins, and how the shares are cut.
struct Place {
    int64_t total, quota;    // length of all items, of a share
    int start;               // what starting an item counts for in its length
    int s, head, qb;         // the item at the position asked for
    int64_t x;               // offset of the position inside that item
    Sequence q;
};

// place, left: a wave's own place in its share while it works on an item (kept in scalar registers they were spilled).
// first, W, len: the sequences, where there are at most 64 of them.
struct PlaceLds { Place place[8]; int64_t left[8]; int first[64], W[64], len[64]; };

// Sum over this lane and those below it, by lane moves inside the vector unit.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved(int64_t x)
{
    const int lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x)
{
    x += moved<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8: inside sixteen lanes
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);      // the last lane of a row of sixteen to the next row (rows 1 and 3)
    x += moved<0x143, 0xc>(x);      // lane 31 to rows 2 and 3
    return x;
}
__device__ __forceinline__ int64_t from_lane(int64_t x, int lane)
{
    const unsigned lo = __builtin_amdgcn_readlane((int)x, lane), hi = __builtin_amdgcn_readlane((int)(x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// The item at position w * quota (false: w is behind the last share).  Every wave computes it for itself, a lane a run of
// sequences: no barrier, and one latency of memory where there are at most 64.
template <typename A>
__device__ __forceinline__ bool find_place(const A &a, int w, Place &p, PlaceLds &lds)
{
    const int lane = threadIdx.x & 63;
    const int run = (a.S + 63) >> 6;
    const int lo = min(lane * run, a.S), hi = min(lo + run, a.S);
    int64_t rows = 0, items = 0;
    Sequence q = {};
    if (run == 1) {
        if (lo < hi) {
            q = sequence_of(a, lo);
            rows = a.HK * rows_before(a, q, q.nqb);
            items = (int64_t)a.HK * q.nqb;
        }
        // (every wave writes the same)
        lds.first[lane] = q.first; lds.W[lane] = q.W; lds.len[lane] = q.len;
    } else {
#pragma unroll 4
        for (int s = lo; s < hi; ++s) {
            const Sequence o = sequence_of(a, s);
            rows += a.HK * rows_before(a, o, o.nqb);
            items += (int64_t)a.HK * o.nqb;
        }
    }
    const int64_t rows_to = wave_scan(rows), items_to = wave_scan(items);
    // Where the chip has more workgroups than there is work for, a start costs less, as no other workgroup waits for the
    // memory it waits for, and shares may be shorter: half of its price (16 sequences of up to 900 rows, 8 key heads x 128: 27
    // -> 22 us; 64 sequences of up to 1000 rows, with it: 41 -> 47).
    const int64_t all = from_lane(rows_to, 63);
    p.start = all < (int64_t)a.shares * a.start ? a.start / 2 : a.start;
    const int64_t sum = rows + items * p.start, upto = rows_to + items_to * p.start;
    p.total = from_lane(upto, 63);
    // any length that no more than `shares` shares of it are needed for
    const int64_t even = (int64_t)((double)p.total * a.per_share) + 1;
    p.quota = uniform(max((even + 63) / 64 * 64, (int64_t)p.start + kShortest));
    const int64_t pos = w * p.quota;
    if (pos >= p.total) return false;
    const uint64_t holds = __builtin_amdgcn_ballot_w64(pos < upto && pos >= upto - sum);
    const int owner = __builtin_ctzll(holds);
    int64_t off = pos - from_lane(upto - sum, owner);
    int s = owner;
    if (run > 1) {
        s = owner * run;
        for (;; ++s) {
            q = sequence_of(a, s);
            const int64_t n = uniform(a.HK * (rows_before(a, q, q.nqb) + (int64_t)q.nqb * p.start));
            if (off < n) break;
            off -= n;
        }
        p.q.first = uniform(q.first); p.q.W = uniform(q.W); p.q.len = uniform(q.len); p.q.nqb = uniform(q.nqb); p.q.before = uniform(q.before);
    } else {
        p.q.first = __builtin_amdgcn_readlane(q.first, owner); p.q.W = __builtin_amdgcn_readlane(q.W, owner);
        p.q.len = __builtin_amdgcn_readlane(q.len, owner); p.q.nqb = __builtin_amdgcn_readlane(q.nqb, owner);
        p.q.before = __builtin_amdgcn_readlane(q.before, owner);
    }
    p.s = s;
    const int64_t head = rows_before(a, p.q, p.q.nqb) + (int64_t)p.q.nqb * p.start;
    p.head = uniform(quotient(off, head));
    off -= p.head * head;
    int lo_b = 0, hi_b = p.q.nqb - 1;          // the last block that begins at or before off
    while (lo_b < hi_b) {
        const int mid = (lo_b + hi_b + 1) >> 1;
        if (rows_before(a, p.q, mid) + (int64_t)mid * p.start <= off) lo_b = mid;
        else hi_b = mid - 1;
    }
    p.qb = uniform(lo_b);
    p.x = uniform(off - rows_before(a, p.q, p.qb) - (int64_t)p.qb * p.start);
    return true;
}

// The item after (s, head, qb); the caller knows that there is one.
template <typename A>
__device__ __forceinline__ void next_item(const A &a, Place &p, const PlaceLds &lds)
{
    p.x = 0;
    if (++p.qb < p.q.nqb) return;
    p.qb = 0;
    if (++p.head < a.HK) return;
    p.head = 0;
    do {
        ++p.s;
        const Sequence q = a.S <= 64 ? complete(a, lds.first[p.s], lds.W[p.s], lds.len[p.s]) : sequence_of(a, p.s);
        p.q.first = uniform(q.first); p.q.W = uniform(q.W); p.q.len = uniform(q.len); p.q.nqb = uniform(q.nqb); p.q.before = uniform(q.before);
    } while (p.q.nqb == 0 && p.s + 1 < a.S);
}

// The items of share w, one after another: work(place, first tile, last tile, whole, slot) for each, and the record of
// the one that the share ends in the middle of.  A cut that would leave no whole tile of an item before it is moved to the
// item's beginning, one that would leave less than kShortest rows behind it to its end, by both of its neighbours alike:
// such a piece would cost more to start than to do, and every piece that is left holds a tile.
template <int BN, typename F>
__device__ __forceinline__ void share_items(int w, PlaceLds &lds, F work)
{
    const int wave = uniform((int)threadIdx.x >> 6);
    ConstPagedArgs &a = *args_again();
    Place p;
    CutItem cut = {};
    if (find_place(a, w, p, lds)) {
        int64_t left = min(p.quota, p.total - w * p.quota);      // to the end of the share, as it was cut
        bool more = true;
        {
            const int64_t n = block_rows(a, p.q, p.qb) + p.start;
            if (p.x < p.start + BN) {
                left += p.x;
                p.x = 0;
            } else if (n - p.x < kShortest) {
                left -= n - p.x;
                more = left > 0;
                if (more) next_item(a, p, lds);
            }
        }
        while (more) {
            ConstPagedArgs &b = *args_again();
            const int start = p.start;
            const int64_t n = block_rows(b, p.q, p.qb) + start, to = p.x + left;
            if (to < n && to < start + BN) break;                // (so p.x is 0) the next share's, from its beginning
            const bool all = n - to < kShortest;                 // up to its end
            const int64_t x1 = all ? n : to;
            const int t0 = tiles_to<BN>(p.x, start), t1 = tiles_to<BN>(x1, start);
            lds.place[wave] = p;
            lds.left[wave] = left;
            work(p, t0, t1, p.x == 0 && all, 2 * w + (p.x == 0));
            asm volatile("" ::: "memory");
            const Place &o = lds.place[wave];
            p.total = uniform(o.total); p.quota = uniform(o.quota); p.start = uniform(o.start);
            p.s = uniform(o.s); p.head = uniform(o.head); p.qb = uniform(o.qb); p.x = uniform(o.x);
            p.q.first = uniform(o.q.first); p.q.W = uniform(o.q.W); p.q.len = uniform(o.q.len);
            p.q.nqb = uniform(o.q.nqb); p.q.before = uniform(o.q.before);
            left = uniform(lds.left[wave]);
            ConstPagedArgs &c = *args_again();
            const int64_t len = block_rows(c, p.q, p.qb) + p.start, end = p.x + left;
            if (end >= len) {
                left = end - len;
                if (left == 0) break;
                next_item(c, p, lds);
                continue;
            }
            if (p.x == 0 && len - end >= kShortest) {            // the cut goes through an item that begins here
                cut.rows = min(c.TB, p.q.W - p.qb * c.TB) * c.G;
                cut.row = p.q.first + p.qb * c.TB;
                cut.head = p.head * c.G;
                cut.parts = quotient(len - kShortest - end, p.quota) + 2;
            }
            break;
        }
    }
    if ((threadIdx.x & 63) == 0) args_again()->cuts[w] = cut;      // (every wave that has this share writes the same)
}

}  // namespace tlin
