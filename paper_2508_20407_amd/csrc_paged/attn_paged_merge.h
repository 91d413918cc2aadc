// Joins the partials of the items that a cut between two shares goes through.
//
// A partial of a row is (O, m, l): O = sum_j 2^(x_j - m) V_j, l = sum_j 2^(x_j - m) over its keys, x_j the logit in base-2
// units.  Over the union of the partials O = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s, M the largest m_s.  The
// workgroups of a share join the item that begins in it and ends in a later one, if there is one.  No atomics: results do
// not depend on who comes first.
#pragma once
#include "share.h"

namespace tlin {

constexpr int kMergeThreads = 256;

// LN threads share a (row, 4 columns): each takes every LN-th partial.  blockIdx.y: which of the item's rows.
template <int DK, int LN>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(const PagedArgs a)
{
    constexpr int TPR = DK / 4;                         // threads across a row
    constexpr int RPB = kMergeThreads / (TPR * LN);     // rows at a time
    __shared__ float red[LN > 1 ? kMergeThreads * 6 : 1];
    const int w = blockIdx.x;
    const CutItem cut = a.cuts[w];
    const int rows = cut.rows, BM = a.BM;
    const int cg = threadIdx.x % TPR, ln = threadIdx.x / TPR % LN, rb = threadIdx.x / (TPR * LN);
    const int c4 = 4 * cg;
    for (int r0 = blockIdx.y * RPB; r0 < rows; r0 += gridDim.y * RPB) {
        const int r = r0 + rb;
        const bool live = r < rows;
        float M = -INFINITY, den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
        constexpr int NB = 4;
        if (live)
            for (int k0 = ln; k0 < cut.parts; k0 += NB * LN) {
                float ms[NB], ls[NB];
                f32x4 os[NB];
#pragma unroll
                for (int e = 0; e < NB; ++e) {
                    ms[e] = -INFINITY;
                    ls[e] = 0.f;
                    os[e] = f32x4{0.f, 0.f, 0.f, 0.f};
                    const int k = k0 + e * LN;
                    if (k >= cut.parts) continue;
                    const int64_t slot = 2 * (int64_t)(w + k) + (k == 0);
                    const int64_t idx = slot * BM + r;
                    ms[e] = a.Mpart[idx];
                    ls[e] = a.Lpart[idx];
                    os[e] = *(const f32x4 *)(a.Opart + idx * DK + c4);
                }
                float Mn = M;
#pragma unroll
                for (int e = 0; e < NB; ++e) Mn = fmaxf(Mn, ms[e]);
                const float w0 = M == -INFINITY ? 0.f : exp2f(M - Mn);
                den *= w0;
                num *= w0;
#pragma unroll
                for (int e = 0; e < NB; ++e) {
                    const float we = ms[e] == -INFINITY ? 0.f : exp2f(ms[e] - Mn);
                    den += we * ls[e];
                    num += we * os[e];
                }
                M = Mn;
            }
        if (LN > 1) {
            __syncthreads();
            float *mine = red + threadIdx.x * 6;
            mine[0] = M; mine[1] = den; mine[2] = num[0]; mine[3] = num[1]; mine[4] = num[2]; mine[5] = num[3];
            __syncthreads();
            if (ln != 0) continue;
#pragma unroll
            for (int k = 1; k < LN; ++k) {
                const float *o = red + (threadIdx.x + k * TPR) * 6;
                const float Mn = fmaxf(M, o[0]);
                const float w1 = M == -INFINITY ? 0.f : exp2f(M - Mn), w2 = o[0] == -INFINITY ? 0.f : exp2f(o[0] - Mn);
                den = w1 * den + w2 * o[1];
                num = w1 * num + w2 * f32x4{o[2], o[3], o[4], o[5]};
                M = Mn;
            }
        }
        if (!live || c4 >= a.D) continue;
        const int tok = r / a.G, hd = cut.head + r - tok * a.G;
        const int64_t row = cut.row + tok;
        const f32x4 o = num * (den > 0.f ? 1.0f / den : den == 0.f ? 0.f : den);      // (not a number stays that)
        const int64_t off = hd * a.o_sh + row * a.o_sr + c4;
        if (a.out_bf16) {
            bf16x4 ob;
#pragma unroll
            for (int e = 0; e < 4; ++e) ob[e] = (__bf16)o[e];
            *(bf16x4 *)((__bf16 *)a.O + off) = ob;
        } else {
            *(f32x4 *)((float *)a.O + off) = o;
        }
        if (a.lse && cg == 0) a.lse[(int64_t)hd * a.T + row] = (M + log2f(den)) * 0.6931471805599453f;
    }
}

}  // namespace tlin
