// Rotary positions, and the append of new rows to a paged cache.
//
// Pair i of a row at position p is turned by the angle p * freqs[i]:
//     y1 = a (x1 cos - x2 sin),    y2 = a (x1 sin + x2 cos).
// Angles are formed and reduced in 64 bits (as turns: p f / 2 pi minus its nearest whole number, so that a
// position of 2^20 keeps all digits of its angle), sine and cosine taken in 64 bits and rounded to fp32 once; the
// turn itself is fp32, rounded to the rows' type once at the end.
//
// Bound by HBM: every row is read once and written once.  A workgroup takes TB tokens with all their heads, so that the
// sines of a token are computed once for all heads (64 pairs: one per thread for four tokens) and kept in LDS; a thread then
// moves 16-byte pieces: both pieces of its pairs where the halves are whole 128-byte lines, else one piece of the row,
// whose columns' partners it finds in LDS, where the lanes of the row leave their pieces.  Loads are non-temporal (4 x 32 heads x
// 8192 rows x 128: 108 -> 101 us), stores where a thread's are whole lines' (131072 rows: 426 -> 407; pieces of lines, 80 columns:
// 85 -> 131 the other way round).
#pragma once
#include "common.h"

namespace tlin {

struct RopeSegment {         // heads of one tensor, rows by token
    const void *x;
    void *y;
    int64_t x_sh, x_sr, y_sh, y_sr;   // element strides; y_sr is not used where rows go to pages
    int32_t H;
};

struct RopeArgs {
    RopeSegment q, k, v;     // q: rotated to dense rows; k: rotated to pages; v: copied to pages (append only)
    int64_t q_sb, qy_sb;     // batch strides (tlin_rope)
    const int32_t *pos;      // tlin_rope: positions [B, rows]
    int64_t pos_stride;
    int32_t rows;            // rows of a batch
    int32_t tokens;          // B * rows, or T
    int32_t TB;              // tokens of a workgroup
    int32_t lanes, vlanes;   // lanes of a row: the units of a rotated row, of a copied row
    int32_t D, rot;
    float amplitude;
    int32_t negate;
    const double *freqs;
    // append
    const int32_t *table, *lens, *starts;
    int32_t S, M, P, lr;     // sequences, table width, pages, log2 of the page's rows
    int32_t table_stride;
    int64_t kp_sp, kp_sr, vp_sp, vp_sr;   // page and row strides of the caches
};

// 16 bytes of a row
template <typename T>
union Pack {
    u32x4 raw;
    T e[16 / sizeof(T)];
};

// Stores a piece; of the last piece of a bf16 row whose D is not whole pieces only the half that belongs to it.
template <typename T>
__device__ __forceinline__ void store_piece(T *at, const Pack<T> &p, int left)
{
    if (left * sizeof(T) < 16) *(u32x2 *)at = u32x2{p.raw[0], p.raw[1]};      // D is a multiple of 4: half of the piece
    else *(u32x4 *)at = p.raw;
}

// What lanes of a wave have written to LDS is there for its other lanes: LDS serves a wave in order, the compiler has to.
__device__ __forceinline__ void wave_step()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// How a row is dealt to threads: both pieces of pairs of halves, a piece of neighbours, a piece of halves by way of LDS.
enum RopeLayout { ROPE_HALVES, ROPE_NEIGHBOURS, ROPE_STAGED };

constexpr int kRopeTokens = 16;      // most tokens of a workgroup
constexpr int kRopePairs = 64;       // most pairs of a row

template <typename T, int LAYOUT, bool APPEND>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a)
{
    constexpr int E = 16 / sizeof(T);           // elements of a piece
    __shared__ float2 cs[kRopeTokens][kRopePairs];
    __shared__ int where[kRopeTokens];          // position
    __shared__ int place[kRopeTokens];          // append: page of the row, or -1
    __shared__ int live[kRopeTokens];
    __shared__ u32x4 stage[LAYOUT == ROPE_STAGED ? 256 : 1];

    const int tid = threadIdx.x;
    const int g0 = blockIdx.x * a.TB;
    const int nt = min(a.TB, a.tokens - g0);
    const int half = a.rot / 2;

    if (tid < nt) {
        if (APPEND) live[tid] = 0;
        else {
            const int g = g0 + tid;
            where[tid] = a.pos[(int64_t)(g / a.rows) * a.pos_stride + g % a.rows];
        }
    }
    __syncthreads();
    if (APPEND) {
        // every sequence that owns some of these tokens says where they go
        for (int s = tid; s < a.S; s += 256) {
            const int first = min(max(a.starts[s], 0), a.tokens), end = min(a.starts[s + 1], a.tokens);
            const int lo = max(first, g0), hi = min(end, g0 + nt);
            if (lo < hi) {
                const int len = (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.M << a.lr);
                for (int g = lo; g < hi; ++g) {
                    const int p = len - (end - g);
                    int page = -1;
                    if (p >= 0) {
                        const int id = a.table[(int64_t)s * a.table_stride + (p >> a.lr)];
                        page = id >= 0 && id < a.P ? id : -1;
                    }
                    where[g - g0] = p;
                    place[g - g0] = page;
                    live[g - g0] = 1;
                }
            }
        }
        __syncthreads();
    }
    for (int i = tid; i < nt * half; i += 256) {
        const int t = i / half, f = i % half;
        if (APPEND && !live[t]) continue;
        const double turns = (double)where[t] * (a.freqs[f] * 0.15915494309189533577);
        double s, c;
        sincospi(2.0 * (turns - rint(turns)), &s, &c);
        cs[t][f] = float2{(float)(c * a.amplitude), (float)(a.negate ? -s * a.amplitude : s * a.amplitude)};
    }
    __syncthreads();

    const int turned = half / E;                // ROPE_HALVES: units that hold pairs, the rest of the row behind them

    // one unit of a rotated row
    auto turn = [&](const T *x, T *y, int t, int u) __attribute__((always_inline)) {
        if (LAYOUT == ROPE_NEIGHBOURS) {
            Pack<T> p;
            p.raw = __builtin_nontemporal_load((const u32x4 *)(x + u * E));
#pragma unroll
            for (int e = 0; e < E; e += 2)
                if (u * E + e < a.rot) {
                    const float2 w = cs[t][(u * E + e) >> 1];
                    const float x1 = (float)p.e[e], x2 = (float)p.e[e + 1];
                    p.e[e] = (T)(x1 * w.x - x2 * w.y);
                    p.e[e + 1] = (T)(x1 * w.y + x2 * w.x);
                }
            store_piece(y + u * E, p, a.D - u * E);
        } else if (LAYOUT == ROPE_STAGED) {
            // columns c below half: x[c] cos - x[c + half] sin; from half to rot: x[c] cos + x[c - half] sin.  The lanes of a
            // row are lanes of one wave: they pass their pieces on through LDS, and in place all have read before one writes.
            const int c = u * E;
            Pack<T> p;
            p.raw = __builtin_nontemporal_load((const u32x4 *)(x + c));
            stage[tid] = p.raw;
            wave_step();
            const T *const row = (const T *)(stage + (tid - u));
            Pack<T> o;
            if (sizeof(T) == 2 && half % 2 == 0) {             // (uniform) pairs of columns have partners side by side
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const int at = c + e < half ? c + e + half : c + e - half;
                    o.raw[e * sizeof(T) / 4] = *(const unsigned *)(row + (c + e < a.rot ? at : 0));
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int at = c + e < half ? c + e + half : c + e - half;
                    o.e[e] = row[c + e < a.rot ? at : 0];
                }
            }
            wave_step();
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (c + e < a.rot) {
                    const bool low = c + e < half;
                    const float2 w = cs[t][low ? c + e : c + e - half];
                    const float own = (float)p.e[e] * w.x, other = (float)o.e[e] * w.y;
                    p.e[e] = (T)(low ? own - other : own + other);
                }
            store_piece(y + c, p, a.D - c);
        } else if (u < turned) {
            Pack<T> p1, p2;
            p1.raw = __builtin_nontemporal_load((const u32x4 *)(x + u * E));
            p2.raw = __builtin_nontemporal_load((const u32x4 *)(x + half + u * E));
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float2 w = cs[t][u * E + e];
                const float x1 = (float)p1.e[e], x2 = (float)p2.e[e];
                p1.e[e] = (T)(x1 * w.x - x2 * w.y);
                p2.e[e] = (T)(x1 * w.y + x2 * w.x);
            }
            __builtin_nontemporal_store(p1.raw, (u32x4 *)(y + u * E));
            __builtin_nontemporal_store(p2.raw, (u32x4 *)(y + half + u * E));
        } else {
            const int col = a.rot + (u - turned) * E;
            Pack<T> p;
            p.raw = __builtin_nontemporal_load((const u32x4 *)(x + col));
            store_piece(y + col, p, a.D - col);
        }
    };
    // f(token, head, unit) over the rows of these tokens: as many whole rows to a wave as it has lanes for, rows that follow
    // each other in memory by following lanes (tokens of a head where `down`: 32 heads of 131072 rows x 128, 407 -> 360 us;
    // 96 columns, twelve lanes of a row among five rows a wave, 82 -> 72)
    auto each = [&](int H, int lanes, bool down, auto f) __attribute__((always_inline)) {
        const int lane = tid & 63, mine = (int)(((float)lane + 0.5f) * (1.0f / (float)lanes)), u = lane - mine * lanes, rows = 64 / lanes;
        if (mine >= rows) return;
        const int n = down ? nt : H;
        const float inv = 1.0f / (float)n;
        for (int r = (tid >> 6) * rows + mine; r < nt * H; r += 4 * rows) {
            // r / n: exact, r is below 2^13 where several tokens share a workgroup (rope_shape), else below 2^20
            const int q = (int)(((float)r + 0.5f) * inv), m = r - q * n;
            f(down ? m : q, down ? q : m, u);
        }
    };
    if (a.q.x)
        each(a.q.H, a.lanes, a.q.y_sr < a.q.y_sh, [&](int t, int h, int u) __attribute__((always_inline)) {
            if (APPEND && !live[t]) return;
            const int g = g0 + t;
            int64_t xo = (int64_t)h * a.q.x_sh, yo = (int64_t)h * a.q.y_sh;
            if (APPEND) {
                xo += (int64_t)g * a.q.x_sr;
                yo += (int64_t)g * a.q.y_sr;
            } else {
                const int b = g / a.rows, r = g % a.rows;
                xo += b * a.q_sb + r * a.q.x_sr;
                yo += b * a.qy_sb + r * a.q.y_sr;
            }
            turn((const T *)a.q.x + xo, (T *)a.q.y + yo, t, u);
        });
    if (APPEND) {
        const int mask = (1 << a.lr) - 1;
        each(a.k.H, a.lanes, a.kp_sr < a.k.y_sh, [&](int t, int h, int u) __attribute__((always_inline)) {
            if (!live[t] || place[t] < 0) return;
            const T *x = (const T *)a.k.x + (int64_t)h * a.k.x_sh + (int64_t)(g0 + t) * a.k.x_sr;
            turn(x, (T *)a.k.y + place[t] * a.kp_sp + h * a.k.y_sh + (where[t] & mask) * a.kp_sr, t, u);
        });
        each(a.v.H, a.vlanes, a.vp_sr < a.v.y_sh, [&](int t, int h, int u) __attribute__((always_inline)) {
            if (!live[t] || place[t] < 0) return;
            const T *x = (const T *)a.v.x + (int64_t)h * a.v.x_sh + (int64_t)(g0 + t) * a.v.x_sr + u * E;
            Pack<T> p;
            p.raw = *(const u32x4 *)x;
            store_piece((T *)a.v.y + place[t] * a.vp_sp + h * a.v.y_sh + (where[t] & mask) * a.vp_sr + u * E, p, a.D - u * E);
        });
    }
}

}  // namespace tlin
