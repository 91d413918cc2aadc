// libtlinattn: entry points of the paged cache (see include/tlinpaged.h).  gfx950 only.
#include "host.h"
#include "attn_paged_bf16.h"
#include "attn_paged_f32.h"
#include "attn_paged_f32_few.h"
#include "attn_paged_merge.h"
#include "pages.h"
#include "rope.h"

using namespace tlin;

namespace {

// ---- rotary positions and append

// Halves of whole 128-byte lines: a thread takes both pieces of its pairs.  Others go through LDS, a thread a piece of the
// row (4 x 32 heads x 8192 rows, rotated columns of D, 36 of 36 at 16384: 115 -> 80 us, 80 of 80 85 -> 66, 64 of 96 95 -> 72,
// and against threads that take pairs of 4 bytes 100 of 128 242 -> 99, 100 of 100 145 -> 92; 131072 rows, 128 of 128: by halves
// 407 when it was 409 to 423 through LDS).
RopeLayout rope_layout(int rot, bool interleaved, int eb)
{
    return interleaved ? ROPE_NEIGHBOURS : rot / 2 * eb % 128 == 0 ? ROPE_HALVES : ROPE_STAGED;
}

// Lanes of a rotated row (one for each of its units: a row is one wave's) and tokens of a workgroup: as many as give each
// thread about four pieces (eight where it takes one at a time: append of 9000 rows, 32 + 8 + 8 heads x 128, 100 columns
// 64 -> 53 us; by halves 46 -> 55), but a thousand workgroups where there are tokens for them (a hundred tokens would
// otherwise sit on a few compute units), and few enough that the kernel's divisions in fp32 are exact.
void rope_shape(RopeArgs &a, RopeLayout layout, int eb, int heads)
{
    const int E = 16 / eb;
    a.lanes = layout == ROPE_HALVES ? a.rot / 2 / E + (a.D - a.rot + E - 1) / E : (a.D + E - 1) / E;
    const int64_t work = (int64_t)heads * a.lanes;
    int64_t tb = (layout == ROPE_HALVES ? 1024 : 2048) / work;
    if (tb > a.tokens / 1024) tb = a.tokens / 1024;
    if (tb > kRopeTokens) tb = kRopeTokens;
    a.TB = tb < 1 ? 1 : (int)tb;
}

template <typename T, bool APPEND>
const void *rope_kernel_for(RopeLayout layout)
{
    return layout == ROPE_HALVES ? (const void *)rope_kernel<T, ROPE_HALVES, APPEND>
           : layout == ROPE_NEIGHBOURS ? (const void *)rope_kernel<T, ROPE_NEIGHBOURS, APPEND> : (const void *)rope_kernel<T, ROPE_STAGED, APPEND>;
}

template <bool APPEND>
tlin_status launch_rope(const RopeArgs &a, int dtype, RopeLayout layout, hipStream_t st)
{
    const int blocks = (a.tokens + a.TB - 1) / a.TB;
    if (blocks >= 1 << 24) return TLIN_ERR_UNSUPPORTED;       // a launch has fewer than 2^32 threads
    tlin_status s = check_device();
    if (s) return s;
    const void *kernel = dtype == TLIN_F32 ? rope_kernel_for<float, APPEND>(layout) : rope_kernel_for<__bf16, APPEND>(layout);
    return launch_kernel(kernel, dim3(blocks), dim3(256), 0, st, a);
}

tlin_status check_rope(const tlin_rope_params *p)
{
    if (p->rot < 2 || p->rot > p->D || p->rot % 2) return TLIN_ERR_INVALID_ARG;
    if (!isfinite(p->amplitude)) return TLIN_ERR_INVALID_ARG;
    return TLIN_OK;
}

// ---- sizes that the paged calls share
// (kernels walk over all sequences, free and fork over pairs of them: a bound on how long that takes)
constexpr int kMaxSequences = 1 << 16;
tlin_status check_paged(const tlin_paged_params *p)
{
    if (!p) return TLIN_ERR_INVALID_ARG;
    if (p->S < 1 || p->T < 1 || p->H < 1 || p->HK < 1 || p->T > kMaxRows) return TLIN_ERR_INVALID_ARG;
    if (p->H % p->HK || p->H / p->HK > 64 || p->H > 1 << 20 || p->S > kMaxSequences) return TLIN_ERR_INVALID_ARG;
    if (!good_dim(p->D)) return TLIN_ERR_UNSUPPORTED;
    if (!good_page_rows(p->page_rows)) return TLIN_ERR_UNSUPPORTED;
    if (p->table_width < 1 || p->num_pages < 1 || (int64_t)p->table_width * p->page_rows > kMaxRows) return TLIN_ERR_INVALID_ARG;
    if (p->max_rows < 1 || p->max_rows > p->T) return TLIN_ERR_INVALID_ARG;
    if (!is_type(p->dtype) || !is_type(p->out_dtype)) return TLIN_ERR_INVALID_ARG;
    if (p->table_stride != 0 && p->table_stride < p->table_width) return TLIN_ERR_INVALID_ARG;
    const int eb = bytes_of(p->dtype);
    tlin_status st;
    if ((st = check_strides(p->kp_stride, p->D, eb)) || (st = check_strides(p->vp_stride, p->D, eb))) return st;
    // a page's rows are addressed from its first byte in 32 bits, pages in 64
    const int64_t most = (int64_t)1 << 32, dense = (int64_t)p->HK * p->page_rows * p->D * eb;
    if (dense >= most || p->kp_stride[0] * eb >= most || p->vp_stride[0] * eb >= most) return TLIN_ERR_INVALID_ARG;
    if (p->kp_stride[2] * eb * p->page_rows >= most || p->vp_stride[2] * eb * p->page_rows >= most) return TLIN_ERR_INVALID_ARG;
    return TLIN_OK;
}

tlin_status check_book(const tlin_book_params *p)
{
    if (!p || p->S < 1 || p->S > kMaxSequences || p->table_width < 1 || p->num_pages < 1 || p->num_pages > kMaxRows) return TLIN_ERR_INVALID_ARG;
    if (!good_page_rows(p->page_rows)) return TLIN_ERR_UNSUPPORTED;
    if ((int64_t)p->table_width * p->page_rows > kMaxRows) return TLIN_ERR_INVALID_ARG;
    if (p->table_stride != 0 && p->table_stride < p->table_width) return TLIN_ERR_INVALID_ARG;
    return TLIN_OK;
}

BookArgs book_args(const tlin_book_params *p)
{
    BookArgs a = {};
    a.S = p->S; a.M = p->table_width; a.P = p->num_pages; a.lr = log2_of(p->page_rows);
    a.stride = p->table_stride ? p->table_stride : p->table_width;
    return a;
}

// ---- attention

// Waves of a workgroup (32 rows each) and what follows from them.
struct PagedShape { int nw, shares, dk, tb; bool few; int bm() const { return few ? kFewRows : nw * 32; } };

int group_of(const tlin_paged_params *p) { return p->H / p->HK; }

// As few waves as hold a sequence's rows, (new row, query head) pairs, up to eight: two at least, so that one loads beside the
// one that computes where rows are few, four where rows of 64 elements leave registers for three workgroups to a
// compute unit.  Shares: the workgroups that the chip holds at once, by registers and LDS (bf16: 64 KB of tiles at
// 128 columns, one workgroup of eight waves or two smaller ones to a compute unit; half of that at 64).
PagedShape paged_shape(const tlin_paged_params *p)
{
    const int64_t rows = (int64_t)p->max_rows * group_of(p);
    const bool bf = p->dtype == TLIN_BF16;
    PagedShape s;
    s.dk = p->D <= 64 ? 64 : 128;
    s.nw = rows <= 64 ? 2 : rows <= 128 || s.dk == 64 || !bf ? 4 : 8;
    s.shares = s.nw == 8 ? kNumCU : s.dk == 128 ? 2 * kNumCU : 3 * kNumCU;
    // up to sixteen fp32 rows: waves on their own, two to a SIMD
    s.few = !bf && rows <= kFewRows;
    if (s.few) {
        s.nw = 4;
        s.shares = 8 * kNumCU;
    }
    s.tb = s.bm() / group_of(p);
    return s;
}

struct PagedWorkspace { float *O, *M, *L; CutItem *cuts; };
size_t workspace_rows(const PagedShape &s) { return 2 * (size_t)s.shares * s.bm(); }
size_t workspace_bytes(const PagedShape &s) { return workspace_rows(s) * (s.dk + 2) * sizeof(float) + s.shares * sizeof(CutItem); }
PagedWorkspace workspace_of(const PagedShape &s, void *ws)
{
    const size_t rows = workspace_rows(s);
    PagedWorkspace w;
    w.O = (float *)ws;
    w.M = w.O + rows * s.dk;
    w.L = w.M + rows;
    w.cuts = (CutItem *)(w.L + rows);
    return w;
}

template <int DU, int NW, bool NT>
tlin_status launch_paged_bf16(const PagedArgs &a, hipStream_t st)
{
    const void *kernel = (const void *)paged_bf16_kernel<DU, NW, NT>;
    constexpr int lds = PagedBf16<DU, NW, NT>::LDS_BYTES;
    static std::atomic<uint64_t> allowed{0};
    tlin_status s = allow_lds(kernel, lds, allowed);
    return s ? s : launch_kernel(kernel, dim3(a.shares), dim3(NW * 64), lds, st, a);
}
template <int DU, int NW, bool TAIL = false>
tlin_status launch_paged_f32(const PagedArgs &a, hipStream_t st)
{
    const void *kernel = (const void *)paged_f32_kernel<DU, NW, TAIL>;
    constexpr int lds = PagedF32<DU, NW>::LDS_BYTES;
    static std::atomic<uint64_t> allowed{0};
    tlin_status s = allow_lds(kernel, lds, allowed);
    return s ? s : launch_kernel(kernel, dim3(a.shares), dim3(NW * 64), lds, st, a);
}
template <int DK>
tlin_status launch_paged_few(const PagedArgs &a, hipStream_t st)
{
    return launch_kernel((const void *)paged_f32_few_kernel<DK>, dim3(a.shares / 4), dim3(256), 0, st, a);
}
template <int DU>
tlin_status launch_paged(const PagedArgs &a, const PagedShape &s, bool bf, bool nt, hipStream_t st)
{
    if constexpr (DU > 32)
        if (!bf && a.D % 32 == 4) return s.nw == 2 ? launch_paged_f32<DU, 2, true>(a, st) : launch_paged_f32<DU, 4, true>(a, st);
    if (!bf) return s.nw == 2 ? launch_paged_f32<DU, 2>(a, st) : launch_paged_f32<DU, 4>(a, st);
    if (s.nw == 2) return nt ? launch_paged_bf16<DU, 2, true>(a, st) : launch_paged_bf16<DU, 2, false>(a, st);
    if (s.nw == 4) return launch_paged_bf16<DU, 4, false>(a, st);
    if constexpr (DU > 64) return launch_paged_bf16<DU, 8, false>(a, st);
    return TLIN_ERR_UNSUPPORTED;      // (not reached: eight waves are for rows of 128)
}

// Threads to a row's partials: eight where there are too few rows to fill the chip with one.
template <int DK>
tlin_status launch_paged_merge(const PagedArgs &a, double items, hipStream_t st)
{
    const int rows = a.TB * a.G;
    const bool many = items * rows * (DK / 4) < kNumCU * 512;
    const void *kernel = many ? (const void *)paged_merge_kernel<DK, 8> : (const void *)paged_merge_kernel<DK, 1>;
    const int rpb = kMergeThreads / (DK / 4) / (many ? 8 : 1);
    int blocks = (rows + rpb - 1) / rpb;
    if (blocks > 16) blocks = 16;
    return launch_kernel(kernel, dim3(a.shares - 1, blocks), dim3(kMergeThreads), 0, st, a);
}

int page_blocks(const tlin_book_params *p) { return (p->num_pages + kPagesPerBlock - 1) / kPagesPerBlock; }

}  // namespace

extern "C" {

tlin_status tlin_rope(const tlin_rope_params *p, const void *x, void *y, const int32_t *pos, const double *freqs, void *stream)
{
    if (!p || p->B < 1 || p->H < 1 || p->rows < 1 || p->H > 1 << 20) return TLIN_ERR_INVALID_ARG;
    if ((int64_t)p->B * p->rows > kMaxRows) return TLIN_ERR_INVALID_ARG;
    if (!good_dim(p->D)) return TLIN_ERR_UNSUPPORTED;
    if (!is_type(p->dtype) || p->pos_stride < 0) return TLIN_ERR_INVALID_ARG;
    tlin_status st = check_rope(p);
    if (st) return st;
    const int eb = bytes_of(p->dtype);
    if ((st = check_strides(p->x_stride, p->D, eb)) || (st = check_strides(p->y_stride, p->D, eb))) return st;
    if (!x || !y || !pos || !freqs) return TLIN_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(pos, 4) || !aligned(freqs, 8)) return TLIN_ERR_INVALID_ARG;
    RopeArgs a = {};
    int64_t xs[3], ys[3];
    const int64_t sizes[2] = {p->H, p->rows}, outer[2] = {p->B, p->H};
    resolve(p->x_stride, sizes, p->D, xs);
    resolve(p->y_stride, sizes, p->D, ys);
    if (written_twice(ys, outer)) return TLIN_ERR_INVALID_ARG;
    if (x == y && (xs[0] != ys[0] || xs[1] != ys[1] || xs[2] != ys[2])) return TLIN_ERR_INVALID_ARG;
    a.q = {x, y, xs[1], xs[2], ys[1], ys[2], p->H};
    a.q_sb = xs[0]; a.qy_sb = ys[0];
    a.pos = pos; a.pos_stride = p->pos_stride;
    a.rows = p->rows; a.tokens = p->B * p->rows;
    a.D = p->D; a.rot = p->rot; a.amplitude = p->amplitude; a.negate = p->transpose != 0;
    a.freqs = freqs;
    const RopeLayout layout = rope_layout(p->rot, p->interleaved != 0, eb);
    rope_shape(a, layout, eb, p->H);
    return launch_rope<false>(a, p->dtype, layout, (hipStream_t)stream);
}

tlin_status tlin_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor, double trained, double slow,
                                  double fast, double *freqs, double *amplitude)
{
    if (rot < 2 || rot % 2 || rot > 128 || !freqs || !(base > 0) || !isfinite(base)) return TLIN_ERR_INVALID_ARG;
    if (scaling < TLIN_ROPE_PLAIN || scaling > TLIN_ROPE_PARTS) return TLIN_ERR_INVALID_ARG;
    if (scaling != TLIN_ROPE_PLAIN && (!(factor >= 1) || !isfinite(factor))) return TLIN_ERR_INVALID_ARG;
    if (scaling == TLIN_ROPE_BASE && rot < 4) return TLIN_ERR_INVALID_ARG;
    if (scaling == TLIN_ROPE_PARTS && (!(trained > 0) || !isfinite(trained) || !(slow >= 0) || !(fast > slow) || !isfinite(fast)))
        return TLIN_ERR_INVALID_ARG;
    if (scaling == TLIN_ROPE_BASE) base *= pow(factor, (double)rot / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = pow(base, -2.0 * i / rot);
        if (scaling == TLIN_ROPE_LINEAR) f /= factor;
        if (scaling == TLIN_ROPE_PARTS) {
            const double turns = f * trained / 6.283185307179586477;
            double keep = (turns - slow) / (fast - slow);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f = f * keep + f / factor * (1 - keep);
        }
        freqs[i] = f;
    }
    if (amplitude) *amplitude = scaling == TLIN_ROPE_PARTS ? 0.1 * log(factor) + 1.0 : 1.0;
    return TLIN_OK;
}

tlin_status tlin_paged_append(const tlin_paged_params *p, const tlin_rope_params *r, const void *q, void *q_out,
                              const void *k, const void *v, void *k_pages, void *v_pages, const int32_t *table,
                              const int32_t *lens, const int32_t *starts, const double *freqs, void *stream)
{
    tlin_status st = check_paged(p);
    if (st) return st;
    const int eb = bytes_of(p->dtype);
    if ((st = check_strides(p->k_stride, p->D, eb)) || (st = check_strides(p->v_stride, p->D, eb))) return st;
    if (!k || !v || !k_pages || !v_pages || !table || !lens || !starts) return TLIN_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(starts, 4)) return TLIN_ERR_INVALID_ARG;
    if (!q != !q_out) return TLIN_ERR_INVALID_ARG;
    RopeArgs a = {};
    bool inter = true;       // nothing is rotated: whole pieces, none of which holds pairs
    a.D = p->D;
    int64_t s1[2], s2[2], s3[3];
    const int64_t rows[1] = {p->T}, page[2] = {p->HK, p->page_rows}, heads[1] = {p->H}, outer[2] = {p->num_pages, p->HK};
    if (r) {
        tlin_rope_params c = *r;
        c.D = p->D;
        if ((st = check_rope(&c))) return st;
        if (!freqs || !aligned(freqs, 8)) return TLIN_ERR_INVALID_ARG;
        inter = r->interleaved != 0;
        a.rot = r->rot; a.amplitude = r->amplitude; a.freqs = freqs;
        if (q) {
            if ((st = check_strides(p->q_stride, p->D, eb)) || (st = check_strides(p->o_stride, p->D, eb))) return st;
            if (!aligned(q, 16) || !aligned(q_out, 16)) return TLIN_ERR_INVALID_ARG;
            resolve(p->q_stride, rows, p->D, s1);
            resolve(p->o_stride, rows, p->D, s2);
            if (written_twice(s2, heads)) return TLIN_ERR_INVALID_ARG;
            if (q == q_out && (s1[0] != s2[0] || s1[1] != s2[1])) return TLIN_ERR_INVALID_ARG;
            a.q = {q, q_out, s1[0], s1[1], s2[0], s2[1], p->H};
        }
    } else if (q) {
        return TLIN_ERR_INVALID_ARG;
    }
    resolve(p->k_stride, rows, p->D, s1);
    resolve(p->kp_stride, page, p->D, s3);
    if (written_twice(s3, outer)) return TLIN_ERR_INVALID_ARG;
    a.k = {k, k_pages, s1[0], s1[1], s3[1], 0, p->HK};
    a.kp_sp = s3[0]; a.kp_sr = s3[2];
    resolve(p->v_stride, rows, p->D, s1);
    resolve(p->vp_stride, page, p->D, s3);
    if (written_twice(s3, outer)) return TLIN_ERR_INVALID_ARG;
    a.v = {v, v_pages, s1[0], s1[1], s3[1], 0, p->HK};
    a.vp_sp = s3[0]; a.vp_sr = s3[2];
    a.table = table; a.lens = lens; a.starts = starts;
    a.S = p->S; a.M = p->table_width; a.P = p->num_pages; a.lr = log2_of(p->page_rows);
    a.table_stride = p->table_stride ? p->table_stride : p->table_width;
    a.tokens = p->T;
    a.vlanes = row_elements(p->D, eb) * eb / 16;
    const RopeLayout layout = rope_layout(a.rot, inter, eb);
    rope_shape(a, layout, eb, (q ? p->H : 0) + 2 * p->HK);
    return launch_rope<true>(a, p->dtype, layout, (hipStream_t)stream);
}

size_t tlin_paged_workspace_bytes(const tlin_paged_params *p)
{
    return check_paged(p) ? 0 : workspace_bytes(paged_shape(p));
}

tlin_status tlin_paged_attn(const tlin_paged_params *p, const void *q, const void *k_pages, const void *v_pages,
                            const int32_t *table, const int32_t *lens, const int32_t *starts, void *O, float *lse, void *ws,
                            size_t ws_bytes, void *stream)
{
    tlin_status st = check_paged(p);
    if (st) return st;
    const float c = p->scale * 1.4426950408889634f;
    if (!(p->scale > 0.f) || !isfinite(c)) return TLIN_ERR_INVALID_ARG;
    if ((st = check_strides(p->q_stride, p->D, bytes_of(p->dtype))) || (st = check_strides(p->o_stride, p->D, bytes_of(p->out_dtype)))) return st;
    if (!q || !k_pages || !v_pages || !table || !lens || !starts || !O) return TLIN_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(O, 16)) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(lse, 4)) return TLIN_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < tlin_paged_workspace_bytes(p)) return TLIN_ERR_WORKSPACE;
    int64_t s2[2], s3[3];
    const int64_t rows[1] = {p->T}, page[2] = {p->HK, p->page_rows}, heads[1] = {p->H};
    resolve(p->o_stride, rows, p->D, s2);
    if (written_twice(s2, heads)) return TLIN_ERR_INVALID_ARG;
    if ((st = check_device())) return st;

    const PagedShape s = paged_shape(p);
    const bool bf = p->dtype == TLIN_BF16;
    PagedArgs a = {};
    const PagedWorkspace w = workspace_of(s, ws);
    a.Q = q; a.K = k_pages; a.V = v_pages;
    a.table = table; a.lens = lens; a.starts = starts;
    a.O = O; a.lse = lse;
    a.Opart = w.O; a.Mpart = w.M; a.Lpart = w.L; a.cuts = w.cuts;
    a.o_sh = s2[0]; a.o_sr = s2[1];
    resolve(p->q_stride, rows, p->D, s2);
    a.q_sh = s2[0]; a.q_sr = s2[1];
    resolve(p->kp_stride, page, p->D, s3);
    a.k_sp = s3[0]; a.k_sh = s3[1]; a.k_sr = s3[2];
    resolve(p->vp_stride, page, p->D, s3);
    a.v_sp = s3[0]; a.v_sh = s3[1]; a.v_sr = s3[2];
    a.S = p->S; a.T = p->T; a.HK = p->HK; a.G = group_of(p);
    a.D = p->D;
    a.M = p->table_width; a.P = p->num_pages; a.lr = log2_of(p->page_rows);
    a.table_stride = p->table_stride ? p->table_stride : p->table_width;
    a.TB = s.tb; a.BM = s.bm();
    a.by_TB.k = 31;
    while ((1 << (a.by_TB.k - 31)) < s.tb) ++a.by_TB.k;
    a.by_TB.m = (uint32_t)((((uint64_t)1 << a.by_TB.k) + s.tb - 1) / s.tb);
    a.shares = s.shares;
    a.per_share = 1.0 / s.shares;
    a.per_G = 1.0f / a.G;
    // What starting an item costs (page ids, queries, first tiles, output), in rows of the cache.  bf16: the prices by which
    // uneven batches came out lowest: 64 sequences of up to 8192 rows, 8 key heads x 128, one row each, 128 / 256 / 512: 190 / 182
    // / 186 us; 2 prompts of 4096 rows, 8 key heads, eight waves, 128 / 256 / 384 / 512: 194 / 164 / 154 / 155.  fp32: no price is
    // ahead of the others by more than where the cuts happen to fall, and 64, the least tried, is taken: 3 windows of up to 250 rows
    // over 9000, 12 heads x 36, 64 / 80 / 96 / 112 / 160: 98 / 101 / 103 / 98 / 97 us; 512 rows over 4096, 32 heads x 128: 325 / 337
    // / 340 / 339 / 328; 16 sequences of up to 20 rows over 4000, 12 heads x 36: 64 / 65 / 68 / 69 / 67; 4 of 300 over 2000, 32
    // heads on 8 x 68: 135 / 129 / 129 / 135 / 140.
    a.start = !bf ? 64 : s.nw == 8 ? 384 : 256;
    a.causal = p->causal != 0;
    a.out_bf16 = p->out_dtype == TLIN_BF16;
    a.scale = p->scale;
    a.c = c;

    const hipStream_t hs = (hipStream_t)stream;
    // Rows that are read once by a call and exceed the last-level cache (256 MB) carry the non-temporal hint, by what the
    // table and the cache can hold of them.
    const int64_t named = (int64_t)p->S * p->table_width, most = named < p->num_pages ? named : p->num_pages;
    const bool nt = p->max_rows <= s.tb && (double)most * p->HK * p->page_rows * p->D * 4 >= 192 << 20;
    const int du = (p->D + 31) / 32 * 32;
    st = s.few ? (s.dk == 64 ? launch_paged_few<64>(a, hs) : launch_paged_few<128>(a, hs))
         : du == 32 ? launch_paged<32>(a, s, bf, nt, hs) : du == 64 ? launch_paged<64>(a, s, bf, nt, hs)
         : du == 96 ? launch_paged<96>(a, s, bf, nt, hs) : launch_paged<128>(a, s, bf, nt, hs);
    if (st) return st;
    const double items = (double)p->S * p->HK * ((p->max_rows + s.tb - 1) / s.tb);
    return s.dk == 64 ? launch_paged_merge<64>(a, items, hs) : launch_paged_merge<128>(a, items, hs);
}

tlin_status tlin_pages_free(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs, const int32_t *seqs,
                            int32_t n, void *stream)
{
    tlin_status st = check_book(p);
    if (st) return st;
    if (n < 0 || n > kMaxSequences || !table || !lens || !refs || (n > 0 && !seqs)) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(refs, 4) || !aligned(seqs, 4)) return TLIN_ERR_INVALID_ARG;
    if (n == 0) return TLIN_OK;
    if ((st = check_device())) return st;
    BookArgs a = book_args(p);
    a.table = table; a.lens = lens; a.refs = refs; a.ids = seqs; a.n = n;
    return launch_kernel((const void *)pages_free_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, a);
}

tlin_status tlin_pages_fork(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs,
                            const int32_t *parents, const int32_t *children, int32_t n, int32_t *status, void *stream)
{
    tlin_status st = check_book(p);
    if (st) return st;
    if (n < 0 || n > kMaxSequences || !table || !lens || !refs || (n > 0 && (!parents || !children || !status))) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(refs, 4) || !aligned(parents, 4) || !aligned(children, 4) || !aligned(status, 4)) return TLIN_ERR_INVALID_ARG;
    if (n == 0) return TLIN_OK;
    if ((st = check_device())) return st;
    BookArgs a = book_args(p);
    a.table = table; a.lens = lens; a.refs = refs; a.ids = parents; a.children = children; a.n = n; a.status = status;
    return launch_kernel((const void *)pages_fork_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, a);
}

// reserve: first and nth_copy [S], fresh [P].  compact: live pages of every block, rank [P], L.
size_t tlin_pages_workspace_bytes(const tlin_book_params *p)
{
    if (check_book(p)) return 0;
    const size_t reserve = 2 * (size_t)p->S + p->num_pages, compact = (size_t)page_blocks(p) + p->num_pages + 1;
    return 4 * (reserve > compact ? reserve : compact);
}

tlin_status tlin_pages_reserve(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs, const int32_t *want,
                               int32_t *moves, int32_t *count, int32_t *status, void *ws, size_t ws_bytes, void *stream)
{
    tlin_status st = check_book(p);
    if (st) return st;
    if (!table || !lens || !refs || !want || !moves || !count || !status) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(refs, 4) || !aligned(want, 4) || !aligned(moves, 4) || !aligned(count, 4) || !aligned(status, 4)) return TLIN_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < tlin_pages_workspace_bytes(p)) return TLIN_ERR_WORKSPACE;
    if ((st = check_device())) return st;
    BookArgs a = book_args(p);
    a.table = table; a.lens = lens; a.refs = refs; a.ids = want; a.moves = moves; a.count = count; a.status = status;
    a.scratch = (int32_t *)ws;
    return launch_kernel((const void *)pages_reserve_kernel, dim3(1), dim3(1024), 0, (hipStream_t)stream, a);
}

tlin_status tlin_pages_compact(const tlin_book_params *p, const int32_t *table, const int32_t *refs, int32_t *table_out,
                               int32_t *refs_out, int32_t *moves, int32_t *count, void *ws, size_t ws_bytes, void *stream)
{
    tlin_status st = check_book(p);
    if (st) return st;
    if (!table || !refs || !table_out || !refs_out || (!moves && p->num_pages > 1) || !count) return TLIN_ERR_INVALID_ARG;
    if (!aligned(table, 4) || !aligned(refs, 4) || !aligned(table_out, 4) || !aligned(refs_out, 4) || !aligned(moves, 4) || !aligned(count, 4)) return TLIN_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < tlin_pages_workspace_bytes(p)) return TLIN_ERR_WORKSPACE;
    if ((st = check_device())) return st;
    BookArgs a = book_args(p);
    a.table_in = table; a.refs_in = refs; a.table = table_out; a.refs = refs_out; a.moves = moves; a.count = count;
    a.scratch = (int32_t *)ws;
    a.nblocks = page_blocks(p);
    const hipStream_t hs = (hipStream_t)stream;
    // Up to 32768 pages every block of the plan counts all of them itself (32 loads a thread that travel together, about
    // 1 us) instead of waiting for a launch of counts (5 us).
    a.counted = p->num_pages > 32768;
    // A book of one block of pages and few table entries is done by the plan's workgroup.
    a.alone = a.nblocks == 1 && (int64_t)p->S * p->table_width <= 16384;
    if (a.counted && (st = launch_kernel((const void *)pages_count_kernel, dim3(a.nblocks), dim3(1024), 0, hs, a))) return st;
    if ((st = launch_kernel((const void *)pages_plan_kernel, dim3(a.nblocks), dim3(1024), 0, hs, a))) return st;
    if (a.alone) return TLIN_OK;
    const int64_t entries = (int64_t)p->S * p->table_width > p->num_pages ? (int64_t)p->S * p->table_width : p->num_pages;
    const int64_t blocks = (entries + 255) / 256;
    return launch_kernel((const void *)pages_apply_kernel, dim3((unsigned)(blocks < 8 * kNumCU ? blocks : 8 * kNumCU)), dim3(256), 0, hs, a);
}

tlin_status tlin_pages_copy(const tlin_cache_params *p, void *a, void *b, const int32_t *moves, const int32_t *count,
                            int32_t max_moves, void *stream)
{
    if (!p || p->layers < 1 || p->num_pages < 1 || p->num_pages > kMaxRows || p->HK < 1 || p->HK > 1 << 20 || !is_type(p->dtype)) return TLIN_ERR_INVALID_ARG;
    if (!good_dim(p->D) || !good_page_rows(p->page_rows)) return TLIN_ERR_UNSUPPORTED;
    const int eb = bytes_of(p->dtype);
    tlin_status st;
    if ((st = check_strides(p->a_stride, p->D, eb))) return st;
    if (b && (st = check_strides(p->b_stride, p->D, eb))) return st;
    if (!aligned(moves, 4) || !aligned(count, 4)) return TLIN_ERR_INVALID_ARG;
    if (!a || !aligned(a, 16) || !aligned(b, 16) || max_moves < 0 || (max_moves > 0 && !moves)) return TLIN_ERR_INVALID_ARG;
    const int64_t sizes[2] = {p->HK, p->page_rows}, outer[2] = {p->num_pages, p->HK};
    int64_t strides[2][3];
    resolve(p->a_stride, sizes, p->D, strides[0]);
    resolve(p->b_stride, sizes, p->D, strides[1]);
    for (int c = 0; c < (b ? 2 : 1); ++c) {
        if (p->layer_stride[c] < 0 || p->layer_stride[c] % (16 / eb) || p->layer_stride[c] >= kMaxBytes / eb) return TLIN_ERR_INVALID_ARG;
        if (p->layers > 1 && !p->layer_stride[c] && strides[c][0] >= kMaxBytes / eb / p->num_pages) return TLIN_ERR_INVALID_ARG;
        if (written_twice(strides[c], outer)) return TLIN_ERR_INVALID_ARG;
    }
    if (max_moves == 0) return TLIN_OK;
    if ((st = check_device())) return st;
    CopyArgs g = {};
    g.moves = moves; g.count = count; g.max_moves = max_moves; g.P = p->num_pages;
    g.layers = p->layers; g.HK = p->HK; g.R = p->page_rows;
    g.caches = b ? 2 : 1;
    const int re = row_elements(p->D, eb);
    g.row_pieces = re * eb / 16;
    g.pieces = (int64_t)p->HK * p->page_rows * g.row_pieces;
    for (int c = 0; c < g.caches; ++c) {
        const int64_t(&s)[3] = strides[c];
        g.cache[c] = (char *)(c == 0 ? a : b);
        g.layer[c] = p->layers == 1 ? 0 : (p->layer_stride[c] ? p->layer_stride[c] : s[0] * p->num_pages) * eb;
        g.page[c] = s[0] * eb; g.head[c] = s[1] * eb; g.row[c] = s[2] * eb;
        // heads outside rows or rows outside heads, without gaps
        g.flat[c] = (s[2] == re && s[1] == (int64_t)re * p->page_rows) || (s[1] == re && s[2] == (int64_t)re * p->HK) || (p->HK == 1 && s[2] == re);
    }
    // 16 KB to a work item: four pieces a thread
    g.parts = (int)((g.pieces + 1023) / 1024);
    const int64_t most = (int64_t)max_moves * g.layers * g.caches * g.parts;
    return launch_kernel((const void *)pages_copy_kernel, dim3((unsigned)(most < 8 * kNumCU ? most : 8 * kNumCU)), dim3(256), 0, (hipStream_t)stream, g);
}

}  // extern "C"
