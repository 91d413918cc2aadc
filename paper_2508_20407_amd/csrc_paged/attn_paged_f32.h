// fp32 attention of new rows over a paged cache, by fp32 matrix instructions (v_mfma_f32_32x32x2_f32).
//
// The same transposed products as in bf16: S^T[key, query] = K Q^T with 32 keys a tile, whose accumulator holds 16 keys of
// one query column a lane, which is the B operand of O^T[d, query] += V^T P^T as it stands: step v of the value product
// contracts keys 8 (v / 4) + v % 4 (lanes 0 to 31) and the same + 4 (lanes 32 to 63), the ones that register v holds.
// The contraction over columns is taken in the order in which 16-byte reads deliver them.  Products, weights and sums
// are fp32 throughout.  Weights are 2^((s - m) c), m the reference point of the row, which moves only where a logit exceeds it
// by 8 base-2 units (any point gives the same result): they reach 256.
//
// Bound by the matrix pipe (157 TFLOP/s): 64 instructions of 64 cycles each for the scores and the values of a tile at 128
// columns, whatever the number of rows in the wave.  Four columns behind whole blocks of 32 (36, 68, 100: TAIL) are summed by
// vector instructions, 64 of 4 cycles in the place of a block's 16 of 64: a lane multiplies its sixteen weights with the four
// values of each key, which all lanes of its half read at one address (3 windows of up to 250 rows over 9000, 12 heads x 36:
// 131 -> 102 us; 512 over 4096, 32 heads x 100: 316 -> 271).
//
// Tiles go to LDS by direct loads, in groups of 16 rows that may lie in different pages, as in attn_paged_bf16.h.  K rows are
// swizzled by row & 15 (16 lanes read 16 bytes of 16 rows at once), V rows by bit 2 of the row (the two halves of a wave
// read rows 4 apart).
#pragma once
#include "attn_bf16.h"
#include "share.h"

namespace tlin {

template <int DU, int NW>
struct PagedF32 {
    static constexpr int DK = DU <= 64 ? 64 : 128;
    static constexpr int BN = 32, BM = NW * 32;
    static constexpr int ROWB = DK * 4, TILE_B = BN * ROWB, CPR = ROWB / 16;
    static constexpr int RPI = 1024 / ROWB;
    static constexpr int NDMA = BN / RPI / NW;
    static constexpr int NGW = NDMA * RPI > 16 ? NDMA * RPI / 16 : 1;
    static constexpr int LDS_BYTES = 4 * TILE_B;
    static_assert(NDMA >= 1 && DU % 32 == 0, "tile does not divide over the waves");
};

template <int DU, int NW, bool TAIL>
__device__ __forceinline__ void paged_f32_item(const Place &p, int t0, int t1, bool direct, int64_t slot)
{
    ConstPagedArgs &a = *args_again();
    using C = PagedF32<DU, NW>;
    constexpr int DK = C::DK, BN = C::BN, BM = C::BM, ROWB = C::ROWB, TILE_B = C::TILE_B, CPR = C::CPR, RPI = C::RPI;
    constexpr int NDMA = C::NDMA, NGW = C::NGW;
    constexpr int DQ = DU / 8, DB = DU / 32 - TAIL;       // 16-byte reads of a key per lane, blocks of 32 output columns

    char *const Ks = tlin_smem;
    char *const Vs = tlin_smem + 2 * TILE_B;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const int j = lane & 31, h = lane >> 5;
    const int nt = t1 - t0;
    const int len = p.q.len, ctx = len - p.q.W;

    // page ids of the group lane % 2 of local tile n
    const int32_t *const row = a.table + (int64_t)p.s * a.table_stride;
    auto load_ids = [&](int n) __attribute__((always_inline)) {
        const int key = (t0 + min(n, nt - 1)) * BN + 16 * (lane & 1);
        return row[min(key >> a.lr, a.M - 1)];
    };
    int idA = load_ids(0), idB = load_ids(1);      // of tile n + 1 and, on its way, n + 2 in iteration n

    // ---- this lane's query row (see attn_paged_bf16.h)
    const int tok0 = p.qb * a.TB;
    const int ntok = min(a.TB, p.q.W - tok0);
    const int r = wave * 32 + j;
    const int tok = (int)(((float)r + 0.5f) * a.per_G), hq = r - tok * a.G;
    const bool mine = tok < ntok;
    const int64_t qrow = p.q.first + tok0 + (mine ? tok : 0);
    const int hd = p.head * a.G + (mine ? hq : 0);
    const int lim = a.causal ? min(len - 1, ctx + tok0 + tok) : len - 1;
    const int wt0 = (int)((wave * 32 + 0.5f) * a.per_G), wt1 = min((int)((wave * 32 + 31.5f) * a.per_G), ntok - 1);
    const int lim0 = uniform(a.causal ? min(len - 1, ctx + tok0 + wt0) : len - 1);
    const int lim1 = uniform(a.causal ? min(len - 1, ctx + tok0 + wt1) : len - 1);
    const int tl = uniform(wt0 >= ntok || lim1 < 0 ? -1 : min(lim1 / BN - t0, nt - 1));

    const int dchunks = a.D >> 2;
    f32x4 qf[DQ];         // columns 8 q + 4 h .. + 3
    {
        const float *qp = (const float *)a.Q + hd * a.q_sh + qrow * a.q_sr + 4 * h;
#pragma unroll
        for (int q = 0; q < DQ; ++q) qf[q] = 8 * q + 4 * h < a.D ? *(const f32x4 *)(qp + 8 * q) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < DQ; ++q) asm volatile("" : "+v"(qf[q]));
    }

    const unsigned k_rb = (unsigned)a.k_sr * 4, v_rb = (unsigned)a.v_sr * 4, kp_b = (unsigned)(a.k_sp * 4), vp_b = (unsigned)(a.v_sp * 4);
    auto kswz = [](int rr) __attribute__((always_inline)) { return rr & 15; };
    auto vswz = [](int rr) __attribute__((always_inline)) { return (rr >> 2 & 1) << 3; };
    unsigned koff[NDMA], voff[NDMA];
#pragma unroll
    for (int i = 0; i < NDMA; ++i) {
        const int drow = (wave * NDMA + i) * RPI + lane / CPR;
        const int kc = (lane % CPR) ^ kswz(drow), vc = (lane % CPR) ^ vswz(drow);
        koff[i] = kc >= dchunks ? kNoChunk : (drow & 15) * k_rb + (kc << 4);
        voff[i] = vc >= dchunks ? kNoChunk : (drow & 15) * v_rb + (vc << 4);
    }
    const unsigned lds_wave = uniform((int)(lds_offset(Ks) + wave * (NDMA * 1024)));
    const char *const Kg = (const char *)a.K + p.head * a.k_sh * 4;
    const char *const Vg = (const char *)a.V + p.head * a.v_sh * 4;
    const int g0 = wave * NDMA * RPI / 16;
    auto missing = [&](int ids, int n) __attribute__((always_inline)) {
        const int key = (t0 + min(n, nt - 1)) * BN + 16 * (lane & 1);
        return (unsigned)(__builtin_amdgcn_ballot_w64(key < len && (unsigned)ids >= (unsigned)a.P) & 3);
    };
    auto issue = [&](int ids, int n, int stage) __attribute__((always_inline)) {
        u32x4 kd[NGW], vd[NGW];
#pragma unroll
        for (int g = 0; g < NGW; ++g) {
            const int key = (t0 + n) * BN + 16 * (g0 + g);
            const unsigned id = __builtin_amdgcn_readlane(ids, g0 + g);
            const bool there = id < (unsigned)a.P;
            const unsigned rows = there ? max(min(16, len - key), 0) : 0, pr = key & ((1 << a.lr) - 1);
            const uint64_t pg = there ? id : 0;
            kd[g] = tile_descriptor(Kg + pg * kp_b + pr * k_rb, rows * k_rb);
            vd[g] = tile_descriptor(Vg + pg * vp_b + pr * v_rb, rows * v_rb);
        }
#pragma unroll
        for (int i = 0; i < NDMA; ++i) {
            direct_load_1k(kd[i * RPI / 16], koff[i], lds_wave + stage * TILE_B + i * 1024);
            direct_load_1k(vd[i * RPI / 16], voff[i], lds_wave + (2 + stage) * TILE_B + i * 1024);
        }
    };

    typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
    typedef __attribute__((address_space(3))) const float lds_f32;
    unsigned kaddr[DQ], vaddr[DB];
#pragma unroll
    for (int q = 0; q < DQ; ++q) kaddr[q] = lds_offset(Ks) + j * ROWB + (((2 * q + h) ^ kswz(j)) << 4);
    // V[key][32 db + j], key = 8 (v / 4) + 4 h + v % 4: bit 2 of the row is h
#pragma unroll
    for (int db = 0; db < DB; ++db) vaddr[db] = lds_offset(Vs) + 4 * h * ROWB + (((8 * db + (j >> 2)) ^ (h << 3)) << 4) + 4 * (j & 3);

    const unsigned taddr = lds_offset(Vs) + 4 * h * ROWB + ((8 * DB ^ (h << 3)) << 4);      // the last four columns of the same keys

    f32x16 oacc[DB];
    f32x4 tail = {0.f, 0.f, 0.f, 0.f};      // their sums over this half's keys
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[db][v] = 0.f;
    const float thr = reference_step(a.c);
    const int D = a.D;

    asm volatile("" : "+v"(idA), "+v"(idB));
    unsigned miss = missing(idA, 0);
    issue(idA, 0, 0);
    for (int n = 0; n < nt; ++n) {
        const int st = (n & 1) * TILE_B;
        wait_vmcnt<0>();
        asm volatile("" : "+v"(idB));
        __builtin_amdgcn_s_barrier();
        const unsigned gone = miss;
        idA = idB;
        idB = load_ids(n + 2);
        if (n + 1 < nt) {
            miss = missing(idA, n + 1);
            issue(idA, n + 1, (n + 1) & 1);
        }
        if (n > tl) continue;
        f32x16 S;
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 0.f;
#pragma unroll
        for (int q = 0; q < DQ; ++q) {
            if (q >= DQ - 3 && 8 * q >= D) continue;      // (uniform; columns are computed in blocks of 32, contracted in steps of 8)
            const f32x4 kf = *(lds_f32x4 *)(uintptr_t)(kaddr[q] + st);
#pragma unroll
            for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[q][e], S, 0, 0, 0);
        }
        if ((t0 + n + 1) * BN - 1 > lim0 || gone) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = (t0 + n) * BN + 8 * (v >> 2) + 4 * h + (v & 3);
                if (key > lim || (gone >> (v >> 3) & 1)) S[v] = -INFINITY;
            }
        }
        float mx = S[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, S[v]);
        mx = xhalf_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > m + thr) != 0) {
            const float mn = fmaxf(m, mx);
            const float alpha = (mn == -INFINITY) ? 1.f : fast_exp2((m - mn) * a.c);
            l *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) oacc[db][v] *= alpha;
            if (TAIL) tail *= alpha;
            m = mn;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float ls = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            S[v] = fast_exp2((S[v] - ref) * a.c);
            ls += S[v];
        }
        l += ls;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            if (TAIL) {
                const f32x4 vt = *(lds_f32x4 *)(uintptr_t)(taddr + st + (8 * (v >> 2) + (v & 3)) * ROWB);
#pragma unroll
                for (int e = 0; e < 4; ++e) tail[e] = fmaf(S[v], vt[e], tail[e]);
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const float vf = *(lds_f32 *)(uintptr_t)(vaddr[db] + st + (8 * (v >> 2) + (v & 3)) * ROWB);
                oacc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, S[v], oacc[db], 0, 0, 0);
            }
        }
    }

    const float lt = xhalf_sum(l);
    if (TAIL)
#pragma unroll
        for (int e = 0; e < 4; ++e) tail[e] = xhalf_sum(tail[e]);
    ConstPagedArgs &z = *args_again();
    if (mine) {
        const float inv = !direct ? 1.f : lt > 0.f ? 1.0f / lt : lt == 0.f ? 0.f : lt;
        const int64_t off = hd * z.o_sh + qrow * z.o_sr;
        float *op = z.Opart + (slot * BM + r) * DK;
        auto put = [&](int d, f32x4 o) __attribute__((always_inline)) {
            o *= inv;
            if (!direct) {
                *(f32x4 *)(op + d) = o;
            } else if (d < z.D) {
                if (z.out_bf16) {
                    bf16x4 ob;
#pragma unroll
                    for (int e = 0; e < 4; ++e) ob[e] = (__bf16)o[e];
                    *(bf16x4 *)((__bf16 *)z.O + off + d) = ob;
                } else {
                    *(f32x4 *)((float *)z.O + off + d) = o;
                }
            }
        };
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                put(32 * db + 8 * g + 4 * h, f32x4{oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2], oacc[db][4 * g + 3]});
        if (TAIL && h == 0) put(32 * DB, tail);
        if (h == 0) {
            if (!direct) {
                z.Mpart[slot * BM + r] = m * z.c;
                z.Lpart[slot * BM + r] = lt;
            } else if (z.lse) {
                z.lse[(int64_t)hd * z.T + qrow] = m * z.scale + logf(lt);
            }
        }
    }
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
}

template <int DU, int NW, bool TAIL>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 8)))
void paged_f32_kernel(const PagedArgs)
{
    using C = PagedF32<DU, NW>;
    __shared__ PlaceLds lds;
    share_items<C::BN>(xcd_remap(blockIdx.x, gridDim.x), lds, [](const Place &p, int t0, int t1, bool whole, int64_t slot) __attribute__((always_inline)) {
        paged_f32_item<DU, NW, TAIL>(p, t0, t1, whole, slot);
    });
}

}  // namespace tlin
