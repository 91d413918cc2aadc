// fp32 attention of few rows over a paged cache: sixteen (new row, query head) pairs a key head at most, a step of single
// tokens most often.
//
// Bound by HBM: a key's row is read for up to sixteen rows only.  On 32-row tiles fed through LDS, where all waves of a
// workgroup share the keys, one wave did all the products and a step ran at 2.3 TB/s.  Here a wave is a share of its
// own: it streams K and V rows from memory into the operand layout of v_mfma_f32_16x16x4_f32, without LDS, barriers or
// other waves to wait for, sixteen keys a tile (one group of rows of one page), the next tile's loads in flight while
// a tile is computed.
//
// Operands.  Scores S^T[key, row] = K Q^T: lane (i, g) = (lane % 16, lane / 16) holds, of key i, columns 16 q + 4 g + e of
// step (q, e): one 16-byte load is the operand of four steps.  The accumulator holds keys 4 g + v of row i in register v, and
// weights are the B operand of O^T[d, row] += V^T P^T as they stand, step s contracting keys 4 g + s.  Its A operand: lane
// (i, g) loads columns 64 b + 4 i .. + 3 of key 4 g + s, whose element e belongs to the block (b, e) of columns 64 b + 4 i + e; a
// lane then ends with four columns in a row, 64 b + 16 g + 4 v + e.
// Products, weights and sums are fp32, in the order of the keys of a share.
#pragma once
#include "attn_bf16.h"
#include "share.h"

namespace tlin {

constexpr int kFewRows = 16;

// One wave-wide load of 16 bytes a lane through a descriptor: offsets at or beyond its size arrive as zeros.
__device__ __forceinline__ f32x4 load_piece(__amdgpu_buffer_rsrc_t r, unsigned offset)
{
    constexpr int kNonTemporal = 2;
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, kNonTemporal);
    return __builtin_bit_cast(f32x4, x);
}

// the largest of the four lanes that hold a row
__device__ __forceinline__ float row_lanes_max(float x)
{
    const unsigned a = __builtin_bit_cast(unsigned, x);
    auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    return xhalf_max(fmaxf(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)));
}

// DK: 64 or 128, a.D at most.
template <int DK>
__device__ __forceinline__ void paged_f32_few_item(const Place &p, int t0, int t1, bool whole, int64_t slot)
{
    constexpr int NQ = DK / 16, NB = DK / 64, BN = 16;
    ConstPagedArgs &a = *args_again();
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int len = p.q.len, ctx = len - p.q.W, D = a.D;
    const int32_t *const row = a.table + (int64_t)p.s * a.table_stride;

    // page ids of tiles 64 j + lane: of the tiles now, and of the next 64
    auto load_ids = [&](int n) __attribute__((always_inline)) { return row[min((t0 + n + lane) * BN >> a.lr, a.M - 1)]; };
    int ids = load_ids(0), idsN = load_ids(64);

    const int tok0 = p.qb * a.TB, ntok = min(a.TB, p.q.W - tok0);
    const int tok = (int)(((float)i + 0.5f) * a.per_G), hq = i - tok * a.G;
    const bool mine = tok < ntok;
    const int64_t qrow = p.q.first + tok0 + (mine ? tok : 0);
    const int hd = p.head * a.G + (mine ? hq : 0);
    const int lim = a.causal ? min(len - 1, ctx + tok0 + tok) : len - 1;
    const int lim0 = a.causal ? min(len - 1, ctx + tok0) : len - 1, lim1 = a.causal ? min(len - 1, ctx + tok0 + ntok - 1) : len - 1;
    const int nt = min(t1 - t0, (lim1 >> 4) + 1 - t0);         // tiles that hold keys some row sees (may be none)

    f32x4 qf[NQ];
    const float *qp = (const float *)a.Q + hd * a.q_sh + qrow * a.q_sr + 4 * g;
#pragma unroll
    for (int q = 0; q < NQ; ++q) qf[q] = 16 * q + 4 * g < D ? *(const f32x4 *)(qp + 16 * q) : f32x4{0.f, 0.f, 0.f, 0.f};

    const unsigned k_rb = (unsigned)a.k_sr * 4, v_rb = (unsigned)a.v_sr * 4, kp_b = (unsigned)(a.k_sp * 4), vp_b = (unsigned)(a.v_sp * 4);
    const char *const Kg = (const char *)a.K + p.head * a.k_sh * 4;
    const char *const Vg = (const char *)a.V + p.head * a.v_sh * 4;
    unsigned koff[NQ], voff[4][NB];
#pragma unroll
    for (int q = 0; q < NQ; ++q) koff[q] = 16 * q + 4 * g < D ? i * k_rb + 64 * q + 16 * g : kNoChunk;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) voff[s][b] = 64 * b + 4 * i < D ? (4 * g + s) * v_rb + 256 * b + 16 * i : kNoChunk;

    struct Tile { f32x4 k[NQ], v[4][NB]; };
    const int P = a.P, lr = a.lr;
    // tile n (below nt), whose page id is in `ids`; whether its page is missing
    auto load = [&](Tile &x, int n) __attribute__((always_inline)) {
        const int key = (t0 + n) * BN;
        const unsigned id = __builtin_amdgcn_readlane(ids, n & 63);
        const bool there = id < (unsigned)P;
        const unsigned rows = there ? min(16, len - key) : 0, pr = key & ((1 << lr) - 1);
        const uint64_t pg = there ? id : 0;
        const auto kd = __builtin_amdgcn_make_buffer_rsrc((void *)(Kg + pg * kp_b + pr * k_rb), 0, (int)(rows * k_rb), 0x00020000);
        const auto vd = __builtin_amdgcn_make_buffer_rsrc((void *)(Vg + pg * vp_b + pr * v_rb), 0, (int)(rows * v_rb), 0x00020000);
#pragma unroll
        for (int q = 0; q < NQ; ++q) x.k[q] = load_piece(kd, koff[q]);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int b = 0; b < NB; ++b) x.v[s][b] = load_piece(vd, voff[s][b]);
        return !there;
    };

    f32x4 O[NB][4];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) O[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = a.c, thr = reference_step(c);
    auto compute = [&](const Tile &x, int n, bool gone) __attribute__((always_inline)) {
        const int key = (t0 + n) * BN;
        f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (q >= NQ - 3 && 16 * q >= D) continue;          // (uniform)
#pragma unroll
            for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[q][e], qf[q][e], S, 0, 0, 0);
        }
        if (key + BN - 1 > lim0 || gone) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (key + 4 * g + v > lim || gone) S[v] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(S[0], S[1]), fmaxf(S[2], S[3]));
        // the reference point moves only where a logit exceeds it by 8 base-2 units (any point gives the same result)
        if (__builtin_amdgcn_ballot_w64(mx > m + thr) != 0) {
            mx = row_lanes_max(mx);
            const float mn = fmaxf(m, mx);
            const float alpha = (mn == -INFINITY) ? 1.f : fast_exp2((m - mn) * c);
            l *= alpha;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[b][e] *= alpha;
            m = mn;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int v = 0; v < 4; ++v) S[v] = fast_exp2((S[v] - ref) * c);
        l += (S[0] + S[1]) + (S[2] + S[3]);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[s][b][e], S[s], O[b][e], 0, 0, 0);
    };
    // ids of the 64 tiles from n on (n a multiple of 64)
    auto turn_ids = [&](int n) __attribute__((always_inline)) {
        if (n > 0 && (n & 63) == 0) {
            ids = idsN;
            idsN = load_ids(n + 64);
        }
    };

    if (nt > 0) {
        Tile A, B;
        bool goneA = load(A, 0), goneB = false;
        for (int n = 0; n < nt; n += 2) {
            if (n + 1 < nt) goneB = load(B, n + 1);            // (an odd tile: its ids are those of the even one before)
            compute(A, n, goneA);
            if (n + 1 >= nt) break;
            turn_ids(n + 2);
            if (n + 2 < nt) goneA = load(A, n + 2);
            compute(B, n + 1, goneB);
        }
    }

    float lt = l + __shfl_xor(l, 16);
    lt += __shfl_xor(lt, 32);
    if (!mine) return;
    ConstPagedArgs &z = *args_again();
    const float inv = !whole ? 1.f : lt > 0.f ? 1.0f / lt : lt == 0.f ? 0.f : lt;
    const int64_t off = hd * z.o_sh + qrow * z.o_sr;
    float *op = z.Opart + (slot * kFewRows + i) * DK;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int d = 64 * b + 16 * g + 4 * v;
            f32x4 o = {O[b][0][v], O[b][1][v], O[b][2][v], O[b][3][v]};
            o *= inv;
            if (!whole) {
                *(f32x4 *)(op + d) = o;
            } else if (d < D) {
                if (z.out_bf16) {
                    bf16x4 ob;
#pragma unroll
                    for (int e = 0; e < 4; ++e) ob[e] = (__bf16)o[e];
                    *(bf16x4 *)((__bf16 *)z.O + off + d) = ob;
                } else {
                    *(f32x4 *)((float *)z.O + off + d) = o;
                }
            }
        }
    if (g == 0) {
        if (!whole) {
            z.Mpart[slot * kFewRows + i] = m * z.c;
            z.Lpart[slot * kFewRows + i] = lt;
        } else if (z.lse) {
            z.lse[(int64_t)hd * z.T + qrow] = m * z.scale + logf(lt);
        }
    }
}

template <int DK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8)))
void paged_f32_few_kernel(const PagedArgs)
{
    __shared__ PlaceLds lds;
    const int w = xcd_remap(blockIdx.x, gridDim.x) * 4 + uniform((int)threadIdx.x >> 6);
    share_items<16>(w, lds, [](const Place &p, int t0, int t1, bool whole, int64_t slot) __attribute__((always_inline)) {
        paged_f32_few_item<DK>(p, t0, t1, whole, slot);
    });
}

}  // namespace tlin
