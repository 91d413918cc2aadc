// bf16 attention of new rows over a paged cache, on the matrix cores.
//
// The pipeline inside a wave, the operand mapping and the LDS layout are those of the dense kernel (attn_bf16_pipe.h):
// transposed scores S^T = K Q^T on v_mfma_f32_32x32x16_bf16 with two score accumulators, so that the softmax
// arithmetic of tile n runs under the score products of tile n + 1 and the value products of tile n; K and V tiles of 64
// rows by direct loads into a ring of two stages, swizzled on the source side; the reference point of a row moves only
// where a logit exceeds it by 8 base-2 units; row sums in fp32 from the fp32 weights, which are rounded to bf16 for the
// value product alone, whose operands are of one type: a weight is off by 2^-8 of itself at most, by
// 1.66e-3 in the root mean square, and so is a sum over values of either sign (2.1 to 2.4e-3 with a bf16 result's own rounding, which
// alone is 1.7e-3).
//
// What paging changes:
//   - Rows come from pages of 16 or more rows, so a tile is four groups of 16 rows that lie anywhere.  A direct load covers 4
//     or 8 rows, never two groups: it takes its group's page through a buffer descriptor of its own, whose size ends
//     with the sequence (what a page holds behind it, NaNs perhaps, arrives as zeros).  Page ids are read four tiles
//     ahead, by lanes 0 to 3, with an ordinary load whose arrival the tile's own wait covers: a scalar load would make the
//     LDS reads of a whole phase wait for it (both count on lgkmcnt and scalar loads return out of order).
//   - The 32 query columns of a wave are (new row, query head) pairs that share a key head, rows outside: the cache is read
//     once for all heads of a group, and a single new row of 8 heads already fills a quarter of the tile.
//   - A workgroup computes the items of its share one after another (share.h).
#pragma once
#include "attn_bf16.h"
#include "share.h"

namespace tlin {


// The lane, computed again from here on.
__device__ __forceinline__ int lane_again()
{
    int ones = -1;
    asm volatile("" : "+v"(ones));
    return __builtin_amdgcn_mbcnt_hi(ones, __builtin_amdgcn_mbcnt_lo(ones, 0));
}
// A (new row, query head) pair of a block: the pair, whether there is one, its row and head, the last key it sees.
struct QueryRow { int r; bool mine; int64_t row; int head, lim; };

// DU: columns computed, at least a.D (32, 64: rows of 64 elements in LDS; 96, 128: of 128).  NT: non-temporal tile loads.
template <int DU, int NW, bool NT>
struct PagedBf16 {
    static constexpr int DK = DU <= 64 ? 64 : 128;
    static constexpr int BN = 64, BM = NW * 32;
    static constexpr int ROWB = DK * 2, TILE_B = BN * ROWB, CPR = ROWB / 16;
    static constexpr int RPI = 1024 / ROWB;         // rows of a direct load
    static constexpr int NDMA = BN / RPI / NW;      // direct loads of a wave per tensor and tile
    static constexpr int DS = DU / 16, DB = DU / 32;
    static constexpr int NGW = NDMA * RPI > 16 ? NDMA * RPI / 16 : 1;   // groups of 16 rows that a wave loads from
    static constexpr int LDS_BYTES = 4 * TILE_B;
    static_assert(NDMA >= 1 && DU % 32 == 0, "tile does not divide over the waves");
};

template <int DU, int NW, bool NT>
__device__ __forceinline__ void paged_bf16_item(const Place &p, int t0, int t1, bool direct, int64_t slot)
{
    ConstPagedArgs &a = *args_again();
    using C = PagedBf16<DU, NW, NT>;
    constexpr int DK = C::DK, BN = C::BN, BM = C::BM, ROWB = C::ROWB, TILE_B = C::TILE_B, CPR = C::CPR, RPI = C::RPI;
    constexpr int NDMA = C::NDMA, DS = C::DS, DB = C::DB, NGW = C::NGW;
    constexpr int VPQ = 29;        // vector instructions per quarter of a tile's weights

    char *const Ks = tlin_smem;
    char *const Vs = tlin_smem + 2 * TILE_B;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const int j = lane & 31, h = lane >> 5;
    const int nt = t1 - t0;
    const int len = p.q.len, ctx = len - p.q.W;

    // ---- page ids: of the group lane % 4 of local tile n, as the table has them
    const int32_t *const row = a.table + (int64_t)p.s * a.table_stride;
    auto load_ids = [&](int n) __attribute__((always_inline)) {
        const int key = (t0 + min(n, nt - 1)) * BN + 16 * (lane & 3);
        return row[min(key >> a.lr, a.M - 1)];
    };
    const int id0 = load_ids(0), id1 = load_ids(1);
    int idB = load_ids(2), idC = load_ids(3);      // of tiles n + 2 and n + 3 during step n (the latter on its way until its top)

    // ---- this lane's query row: (new row, query head) pair r of the block.  Computed where it is needed, for the queries, a
    // mask and the output, and not kept through the loop, whose registers are all taken.
    const int tok0 = p.qb * a.TB;                              // first new row of the block
    const int ntok = min(a.TB, p.q.W - tok0);
    const int first = p.q.first, head = p.head;
    auto query_row = [=](const auto &b) __attribute__((always_inline)) {
        QueryRow x;
        x.r = wave * 32 + (lane_again() & 31);
        const int G = b.G, tok = (int)(((float)x.r + 0.5f) * b.per_G), hq = x.r - tok * G;
        x.mine = tok < ntok;
        x.row = first + tok0 + (x.mine ? tok : 0);
        x.head = head * G + (x.mine ? hq : 0);
        x.lim = b.causal ? min(len - 1, ctx + tok0 + tok) : len - 1;
        return x;
    };
    // of the wave: first and last limit of its rows; the last tile it computes on, or -1
    const int wt0 = (int)((wave * 32 + 0.5f) * a.per_G), wt1 = min((int)((wave * 32 + 31.5f) * a.per_G), ntok - 1);
    const int lim0 = uniform(a.causal ? min(len - 1, ctx + tok0 + wt0) : len - 1);
    const int lim1 = uniform(a.causal ? min(len - 1, ctx + tok0 + wt1) : len - 1);
    const int tl = uniform(wt0 >= ntok || lim1 < 0 ? -1 : min(lim1 / BN - t0, nt - 1));

    const int dchunks = (a.D + 7) >> 3;
    bf16x8 qf[DS];
    {
        const QueryRow x = query_row(a);
        const __bf16 *qp = (const __bf16 *)a.Q + x.head * a.q_sh + x.row * a.q_sr + 8 * h;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            const int keep = a.D - 16 * s - 8 * h;             // columns of this fragment that exist
            if (keep <= 0) { qf[s] = bf16x8{}; continue; }
            u32x4 u = *(const u32x4 *)(qp + 16 * s);
            if (keep < 8) u[2] = u[3] = 0;                     // (D is a multiple of 4)
            qf[s] = __builtin_bit_cast(bf16x8, u);
        }
    }

    // ---- tile loads.  Load i of this wave covers tile rows (wave * NDMA + i) * RPI ..; this lane lands on row drow, chunk
    // position lane % CPR, and fetches chunk (lane % CPR) ^ swz(row); offsets count from the row's group of 16
    const unsigned k_rb = (unsigned)a.k_sr * 2, v_rb = (unsigned)a.v_sr * 2, kp_b = (unsigned)(a.k_sp * 2), vp_b = (unsigned)(a.v_sp * 2);
    unsigned koff[NDMA], voff[NDMA];
#pragma unroll
    for (int i = 0; i < NDMA; ++i) {
        const int drow = (wave * NDMA + i) * RPI + lane / CPR;
        const int kc = (lane % CPR) ^ Swz<DK>::k(drow), vc = (lane % CPR) ^ Swz<DK>::v(drow);
        koff[i] = kc >= dchunks ? kNoChunk : (drow & 15) * k_rb + (kc << 4);
        voff[i] = vc >= dchunks ? kNoChunk : (drow & 15) * v_rb + (vc << 4);
    }
    const unsigned lds_wave = uniform((int)(lds_offset(Ks) + wave * (NDMA * 1024)));
    const char *const Kg = (const char *)a.K + p.head * a.k_sh * 2;
    const char *const Vg = (const char *)a.V + p.head * a.v_sh * 2;
    // groups of local tile n whose rows exist but whose page does not (bits 0 to 3)
    auto missing = [&](int ids, int n) __attribute__((always_inline)) {
        const int key = (t0 + min(n, nt - 1)) * BN + 16 * (lane & 3);
        return (unsigned)(__builtin_amdgcn_ballot_w64(key < len && (unsigned)ids >= (unsigned)a.P) & 15);
    };
    // Of the 16 rows of group g of local tile n: page and row in 32-bit bytes (the host bounds the strides), as many
    // bytes as there are rows below the sequence's end, none where the page is missing.
    auto descriptor = [&](const char *base, unsigned page_bytes, unsigned rb, int ids, int n, int g) __attribute__((always_inline)) {
        const int key = (t0 + min(n, nt - 1)) * BN + 16 * g;
        const unsigned id = __builtin_amdgcn_readlane(ids, g);
        const bool there = id < (unsigned)a.P;
        const unsigned rows = there ? max(min(16, len - key), 0) : 0;
        return tile_descriptor(base + (uint64_t)(there ? id : 0) * page_bytes + (key & ((1 << a.lr) - 1)) * rb, rows * rb);
    };
    const int g0 = wave * NDMA * RPI / 16;                     // first group of this wave
    struct Desc { u32x4 d[NGW]; };
    auto descriptors_k = [&](int ids, int n) __attribute__((always_inline)) {
        Desc x;
#pragma unroll
        for (int g = 0; g < NGW; ++g) x.d[g] = descriptor(Kg, kp_b, k_rb, ids, n, g0 + g);
        return x;
    };
    auto descriptors_v = [&](int ids, int n) __attribute__((always_inline)) {
        Desc x;
#pragma unroll
        for (int g = 0; g < NGW; ++g) x.d[g] = descriptor(Vg, vp_b, v_rb, ids, n, g0 + g);
        return x;
    };
    auto dma_k = [&](const Desc &x, int i, int stage) __attribute__((always_inline)) {
        direct_load_1k<NT>(x.d[i * RPI / 16], koff[i], lds_wave + stage * TILE_B + i * 1024);
    };
    auto dma_v = [&](const Desc &x, int i, int stage) __attribute__((always_inline)) {
        direct_load_1k<NT>(x.d[i * RPI / 16], voff[i], lds_wave + (2 + stage) * TILE_B + i * 1024);
    };
    // D not a multiple of 8: clears columns D .. of the chunk that straddles D in the K rows that this wave loaded
    auto scrub = [&](int stage) __attribute__((always_inline)) {
        if (!(a.D & 7)) return;
        if (lane < NDMA * RPI) {
            const int rr = wave * NDMA * RPI + lane;
            const int pos = (a.D >> 3) ^ Swz<DK>::k(rr);
            *(u32x2 *)(Ks + stage * TILE_B + rr * ROWB + (pos << 4) + 8) = u32x2{0u, 0u};
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    // ---- loop-invariant LDS addresses
    const int i16 = lane & 15, blk1 = (lane >> 4) & 1;
    unsigned kaddr[DS], vaddr[DB];
#pragma unroll
    for (int s = 0; s < DS; ++s) kaddr[s] = lds_offset(Ks) + j * ROWB + (((2 * s + h) ^ Swz<DK>::k(j)) << 4);
    {
        const int r0 = 4 * h + (i16 >> 2);
        const int sw = Swz<DK>::v(r0) << 4;
#pragma unroll
        for (int db = 0; db < DB; ++db) vaddr[db] = lds_offset(Vs) + r0 * ROWB + ((64 * db + 32 * blk1 + 8 * (i16 & 3)) ^ sw);
    }

    f32x16 oacc[DB];
    float m = -INFINITY, l = 0.f, mc = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[db][v] = 0.f;
    const float thr = reference_step(a.c);
    bf16x8 pb[2][2];
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

    auto qk_zero = [&](f32x16 (&S)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int v = 0; v < 16; ++v) S[kk][v] = 0.f;
    };
    auto qk_step = [&](f32x16 (&S)[2], int s, int kk, int kstage) __attribute__((always_inline)) {
        const bf16x8 kf = *(lds_bf16x8 *)(uintptr_t)(kaddr[s] + kstage * TILE_B + kk * (32 * ROWB));
        S[kk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], S[kk], 0, 0, 0);
    };
    auto weights_q = [&](const f32x16 (&S)[2], int kb, int t2) __attribute__((always_inline)) {
        float ls = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = fast_exp2(fmaf(S[kb][8 * t2 + e], a.c, -mc));
            const float p1 = fast_exp2(fmaf(S[kb][8 * t2 + e + 1], a.c, -mc));
            pb[kb][t2][e] = (__bf16)p0;
            pb[kb][t2][e + 1] = (__bf16)p1;
            ls += p0 + p1;
        }
        l += ls;
    };
    // value product number i of a tile (i = 8 kb + 4 t2 + db at 128 columns): its V operand, and the product
    auto v_read = [&](int i, unsigned vbase) __attribute__((always_inline)) {
        const int kb = i / (2 * DB), t2 = (i / DB) % 2, db = i % DB;
        const unsigned ad = vaddr[db] + vbase + (kb * 32 + 16 * t2) * ROWB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)ad);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(ad + 8 * ROWB));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto pv_op = [&](int i, bf16x8 vf) __attribute__((always_inline)) {
        const int kb = i / (2 * DB), t2 = (i / DB) % 2, db = i % DB;
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[kb][t2], oacc[db], 0, 0, 0);
    };
    // keys behind this row's limit, and keys of missing pages
    auto mask = [&](f32x16 (&S)[2], int key0, unsigned miss) __attribute__((always_inline)) {
        const int lim = query_row(*args_again()).lim, h = lane_again() >> 5;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = key0 + kb * 32 + 8 * (v >> 2) + 4 * h + (v & 3);
                if (key > lim || (miss >> (2 * kb + (v >> 3)) & 1)) S[kb][v] = -INFINITY;
            }
        asm volatile("" ::: "memory");
    };
    auto row_max = [&](const f32x16 (&S)[2]) __attribute__((always_inline)) {
        float mx = S[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, S[kb][v]);
        return xhalf_max(mx);
    };
    auto move_reference = [&](float mx) __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(mx > m + thr) != 0) {
            const float mn = fmaxf(m, mx);
            const float alpha = (mn == -INFINITY) ? 1.f : fast_exp2((m - mn) * a.c);
            l *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) oacc[db][v] *= alpha;
            m = mn;
            mc = (m == -INFINITY) ? 0.f : m * a.c;
        }
    };

    // during step n: K(n + 2), V(n + 1), groups of tile n + 1 that are missing
    Desc dk, dv;
    unsigned miss;
    // The top of step n: this wave's loads have landed, and every wave has left the stages that K(n + 2) and V(n + 1) go to.
    auto top = [&](int n, int kst) __attribute__((always_inline)) {
        wait_vmcnt<0>();
        asm volatile("" : "+v"(idC));
        scrub(kst);
        __builtin_amdgcn_s_barrier();
    };
    // what step n + 1 loads; the ids of tile n + 4 set out
    auto advance = [&](int n) __attribute__((always_inline)) {
        dk = descriptors_k(idC, n + 3);
        dv = descriptors_v(idB, n + 2);
        miss = missing(idB, n + 2);
        idB = idC;
    };

    constexpr int KPF = 4, VPF = 2, WA = 2;     // reads ahead of K and V operands, quarters of the weights in phase A
    auto step = [&](const f32x16 (&Sc)[2], f32x16 (&Sn)[2], int n, auto kst, auto vst) __attribute__((always_inline)) {
        constexpr int KST = decltype(kst)::value, VST = decltype(vst)::value;
        top(n, KST);
        // phase A: scores of tile n + 1, half of the weights of tile n, the loads of K(n + 2) and V(n + 1)
        qk_zero(Sn);
#pragma unroll
        for (int s = 0; s < DS; ++s) {
#pragma unroll
            for (int i = (s * 2 * NDMA) / DS; i < ((s + 1) * 2 * NDMA) / DS; ++i) {
                if (i < NDMA) dma_k(dk, i, VST);
                else dma_v(dv, i - NDMA, KST);
            }
            qk_step(Sn, s, 0, KST);
            qk_step(Sn, s, 1, KST);
        }
#pragma unroll
        for (int q = 0; q < WA; ++q) weights_q(Sc, q >> 1, q & 1);
#pragma unroll
        for (int q = 0; q < WA; ++q) asm volatile("" : "+v"(pb[q >> 1][q & 1]));
        asm volatile("" : "+v"(l));
#pragma unroll
        for (int i = 0; i < KPF; ++i) __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 0);
        static_for<2 * DS>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, 1, 0);
            if (i + KPF < 2 * DS) __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 0);
            constexpr int nv = (VPQ * WA * (i + 1)) / (2 * DS) - (VPQ * WA * i) / (2 * DS);
            if (nv > 0) __builtin_amdgcn_sched_group_barrier(SG_VALU | SG_TRANS, nv, 0);
        });
        __builtin_amdgcn_sched_barrier(0);
        if ((t0 + n + 2) * BN - 1 > lim0 || miss) mask(Sn, (t0 + n + 1) * BN, miss);
        const int idN = load_ids(n + 4);
        // phase B: value products of tile n, the rest of its weights, the row maximum of tile n + 1
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) pv_op(i, v_read(i, VST * TILE_B));
#pragma unroll
        for (int q = WA; q < 4; ++q) weights_q(Sc, q >> 1, q & 1);
#pragma unroll
        for (int i = 2 * DB; i < 4 * DB; ++i) pv_op(i, v_read(i, VST * TILE_B));
        const float mx = row_max(Sn);
        // (some 30 scalar instructions a group: behind the barrier, ahead of the first product, they cost a tenth of the step)
        advance(n);
#pragma unroll
        for (int g = 0; g < NGW; ++g) asm volatile("" : "+s"(dk.d[g]), "+s"(dv.d[g]));
        asm volatile("" : "+s"(miss));
#pragma unroll
        for (int i = 0; i < 2 * VPF; ++i) __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 1);
        static_for<4 * DB>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, 1, 1);
            if (i + VPF < 4 * DB) __builtin_amdgcn_sched_group_barrier(SG_DSR, 2, 1);
            constexpr int nv = i < 2 * DB ? (VPQ * (4 - WA) * (i + 1)) / (2 * DB) - (VPQ * (4 - WA) * i) / (2 * DB) : 3;
            if (nv > 0) __builtin_amdgcn_sched_group_barrier(SG_VALU | SG_TRANS, nv, 1);
        });
        __builtin_amdgcn_sched_barrier(0);
        move_reference(mx);
        idC = idN;
    };
    // the top of a step without the pipeline behind it
    auto meet = [&](int n) __attribute__((always_inline)) {
        top(n, (n + 1) & 1);
        const int idN = load_ids(n + 4);
        if (n + 1 < nt) {
#pragma unroll
            for (int i = 0; i < NDMA; ++i) dma_k(dk, i, n & 1);
#pragma unroll
            for (int i = 0; i < NDMA; ++i) dma_v(dv, i, (n + 1) & 1);
        }
        advance(n);
        idC = idN;
    };

    using st0 = std::integral_constant<int, 0>;
    using st1 = std::integral_constant<int, 1>;
    f32x16 S0[2], S1[2];
    // prologue: K(0), then K(1) and V(0); scores and reference point of tile 0
    {
        int i0 = id0, i1 = id1;
        asm volatile("" : "+v"(i0), "+v"(i1), "+v"(idB), "+v"(idC));      // arrived, before the loads that are counted by hand
        const Desc d0 = descriptors_k(i0, 0), d1 = descriptors_k(i1, 1), e0 = descriptors_v(i0, 0);
        const unsigned miss0 = missing(i0, 0);
        dk = descriptors_k(idB, 2);
        dv = descriptors_v(i1, 1);
        miss = missing(i1, 1);
#pragma unroll
        for (int i = 0; i < NDMA; ++i) dma_k(d0, i, 0);
        if (nt > 1) {
#pragma unroll
            for (int i = 0; i < NDMA; ++i) dma_k(d1, i, 1);
        }
#pragma unroll
        for (int i = 0; i < NDMA; ++i) dma_v(e0, i, 0);
        // the queries, requested before the tiles, are waited for with them: one latency instead of two
#pragma unroll
        for (int s = 0; s < DS; ++s) asm volatile("" : "+v"(qf[s]));
        wait_vmcnt<0>();
        scrub(0);
        __builtin_amdgcn_s_barrier();
        if (tl >= 0) {
            qk_zero(S0);
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                qk_step(S0, s, 0, 0);
                qk_step(S0, s, 1, 0);
            }
#pragma unroll
            for (int i = 0; i < KPF; ++i) __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 2);
            static_for<2 * DS>([&](auto ic) __attribute__((always_inline)) {
                __builtin_amdgcn_sched_group_barrier(SG_MFMA, 1, 2);
                if (decltype(ic)::value + KPF < 2 * DS) __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 2);
            });
            __builtin_amdgcn_sched_barrier(0);
            if ((t0 + 1) * BN - 1 > lim0 || miss0) mask(S0, t0 * BN, miss0);
            move_reference(row_max(S0));
        }
    }
    int n = 0;
    for (; n + 1 < tl; n += 2) {
        step(S0, S1, n, st1{}, st0{});
        step(S1, S0, n + 1, st0{}, st1{});
    }
    if (n < tl) {
        step(S0, S1, n, st1{}, st0{});
        ++n;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) S0[kk] = S1[kk];
    }
    // the wave's last tile: weights and value products only
    if (tl >= 0) {
        meet(n);
        const unsigned vbase = (n & 1) * TILE_B;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            weights_q(S0, kb, 0);
            weights_q(S0, kb, 1);
#pragma unroll
            for (int i = 2 * DB * kb; i < 2 * DB * (kb + 1); ++i) pv_op(i, v_read(i, vbase));
        }
        ++n;
    }
    for (; n < nt; ++n) meet(n);
    // the ring is free for the next item once every wave is here and nothing flies any more; the output is not waited for
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();

    // ---- output.  Accumulator register v of block db is column 32 db + 8 (v / 4) + 4 h + v % 4.
    const float lt = xhalf_sum(l);
    ConstPagedArgs &z = *args_again();
    const QueryRow x = query_row(z);
    const int r = x.r, oh = lane_again() >> 5;
    if (x.mine) {
        if (direct) {
            const float inv = lt > 0.f ? 1.0f / lt : lt == 0.f ? 0.f : lt;      // a row that sees nothing: zeros
            const int64_t off = x.head * z.o_sh + x.row * z.o_sr;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int d = 32 * db + 8 * g + 4 * oh;
                    if (d >= z.D) continue;
                    f32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = oacc[db][4 * g + e] * inv;
                    if (z.out_bf16) {
                        bf16x4 ob;
#pragma unroll
                        for (int e = 0; e < 4; ++e) ob[e] = (__bf16)o[e];
                        *(bf16x4 *)((__bf16 *)z.O + off + d) = ob;
                    } else {
                        *(f32x4 *)((float *)z.O + off + d) = o;
                    }
                }
            if (z.lse && oh == 0) z.lse[(int64_t)x.head * z.T + x.row] = m * z.scale + logf(lt);
        } else {
            float *op = z.Opart + (slot * BM + r) * DK;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = oacc[db][4 * g + e];
                    *(f32x4 *)(op + 32 * db + 8 * g + 4 * oh) = o;
                }
            if (oh == 0) {
                z.Mpart[slot * BM + r] = m * z.c;
                z.Lpart[slot * BM + r] = lt;
            }
        }
    }
}

template <int DU, int NW, bool NT>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(NW < 8 ? 2 : 1, 8)))
void paged_bf16_kernel(const PagedArgs)
{
    using C = PagedBf16<DU, NW, NT>;
    __shared__ PlaceLds lds;
    share_items<C::BN>(xcd_remap(blockIdx.x, gridDim.x), lds, [](const Place &p, int t0, int t1, bool whole, int64_t slot) __attribute__((always_inline)) {
        paged_bf16_item<DU, NW, NT>(p, t0, t1, whole, slot);
    });
}

}  // namespace tlin
