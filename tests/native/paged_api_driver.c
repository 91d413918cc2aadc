/* Host-side checks of the paged cache's entry points, meant to be built together with their source under
 * AddressSanitizer and UndefinedBehaviorSanitizer (host code only) and run on a machine without a GPU: every call below
 * returns before any HIP call. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "tlinpaged.h"

static int fails = 0;
#define CHECK(c) do { if (!(c)) { printf("FAILED line %d: %s\n", __LINE__, #c); ++fails; } } while (0)

static tlin_paged_params paged(void)
{
    tlin_paged_params p;
    memset(&p, 0, sizeof p);
    p.S = 2; p.T = 4; p.H = 4; p.HK = 2; p.D = 64; p.page_rows = 16; p.table_width = 3; p.num_pages = 9; p.max_rows = 2;
    p.dtype = p.out_dtype = TLIN_BF16; p.causal = 1; p.scale = 0.125f;
    return p;
}
static tlin_rope_params rope(void)
{
    tlin_rope_params p;
    memset(&p, 0, sizeof p);
    p.B = p.H = 1; p.rows = 4; p.D = p.rot = 64; p.dtype = TLIN_BF16; p.amplitude = 1.f;
    return p;
}

int main(void)
{
    static char memory[1 << 12];
    void *fake = (void *)(((uintptr_t)memory + 255) / 256 * 256);   /* aligned, never dereferenced */
    double f[64], amplitude;
    const size_t much = (size_t)1 << 40;
    const int64_t far[] = {INT64_MAX, INT64_MAX - 7, (int64_t)1 << 62, (int64_t)1 << 61, (int64_t)1 << 60, (int64_t)1 << 48};

    /* strides near the ends of 64 bits are refused, wherever they stand */
    for (unsigned i = 0; i < sizeof far / sizeof *far; ++i)
        for (int dt = 0; dt < 2; ++dt)
            for (int axis = 0; axis < 3; ++axis) {
                tlin_paged_params p = paged();
                p.dtype = dt;
                const int64_t page[3] = {2048, 1024, 64};
                int64_t *const caches[2] = {p.kp_stride, p.vp_stride};
                for (int c = 0; c < 2; ++c) {
                    memcpy(caches[c], page, sizeof page);
                    caches[c][axis] = far[i];
                    CHECK(tlin_paged_workspace_bytes(&p) == 0);
                    CHECK(tlin_paged_attn(&p, fake, fake, fake, fake, fake, fake, fake, NULL, fake, much, NULL) == TLIN_ERR_INVALID_ARG);
                    CHECK(tlin_paged_append(&p, NULL, NULL, NULL, fake, fake, fake, fake, fake, fake, fake, NULL, NULL) == TLIN_ERR_INVALID_ARG);
                    memset(caches[c], 0, sizeof page);
                }
                if (axis < 2) {
                    int64_t *const rows[4] = {p.q_stride, p.o_stride, p.k_stride, p.v_stride};
                    for (int c = 0; c < 4; ++c) {
                        rows[c][0] = 256; rows[c][1] = 64;
                        rows[c][axis] = far[i];
                        if (c < 2) CHECK(tlin_paged_attn(&p, fake, fake, fake, fake, fake, fake, fake, NULL, fake, much, NULL) == TLIN_ERR_INVALID_ARG);
                        else CHECK(tlin_paged_append(&p, NULL, NULL, NULL, fake, fake, fake, fake, fake, fake, fake, NULL, NULL) == TLIN_ERR_INVALID_ARG);
                        rows[c][0] = rows[c][1] = 0;
                    }
                }
                tlin_rope_params r = rope();
                r.dtype = dt;
                for (int k = 0; k < 3; ++k) r.x_stride[k] = r.y_stride[k] = 64;
                r.x_stride[axis] = far[i];
                CHECK(tlin_rope(&r, fake, fake, fake, (double *)fake, NULL) == TLIN_ERR_INVALID_ARG);
                tlin_cache_params c;
                memset(&c, 0, sizeof c);
                c.layers = 2; c.num_pages = 9; c.HK = 2; c.page_rows = 16; c.D = 64; c.dtype = dt;
                memcpy(c.a_stride, page, sizeof page);
                c.a_stride[axis] = far[i];
                CHECK(tlin_pages_copy(&c, fake, NULL, fake, NULL, 1, NULL) == TLIN_ERR_INVALID_ARG);
                memset(c.a_stride, 0, sizeof page);
                c.layer_stride[0] = far[i];
                CHECK(tlin_pages_copy(&c, fake, NULL, fake, NULL, 1, NULL) == TLIN_ERR_INVALID_ARG);
                /* layers as far apart as their pages say, beyond an address space */
                c.layer_stride[0] = 0;
                c.num_pages = 1 << 30;
                memcpy(c.a_stride, page, sizeof page);
                c.a_stride[0] = (int64_t)1 << 40;
                CHECK(tlin_pages_copy(&c, fake, NULL, fake, NULL, 1, NULL) == TLIN_ERR_INVALID_ARG);
            }

    /* workspaces over the ranges of the sizes */
    static const int Gs[] = {1, 3, 8, 64}, Ws[] = {1, 2, 16, 17, 64, 100, 4096, 1 << 30}, Ds[] = {8, 36, 64, 68, 128};
    for (unsigned g = 0; g < 4; ++g)
        for (unsigned w = 0; w < 8; ++w)
            for (unsigned d = 0; d < 5; ++d)
                for (int hk = 1; hk <= 1 << 14; hk *= 128) {
                    tlin_paged_params p = paged();
                    p.dtype = TLIN_F32;
                    p.T = 1 << 30; p.HK = hk; p.H = hk * Gs[g]; p.D = Ds[d]; p.max_rows = Ws[w]; p.num_pages = INT32_MAX;
                    p.table_width = 1 << 26; p.S = 65536;
                    CHECK(tlin_paged_workspace_bytes(&p) > 0 && tlin_paged_workspace_bytes(&p) < (size_t)1 << 30);
                }
    tlin_book_params b = {65536, 1 << 26, 1 << 30, 16, 0};
    CHECK(tlin_pages_workspace_bytes(&b) >= (size_t)4 << 30);
    b.num_pages = INT32_MAX;
    CHECK(tlin_pages_workspace_bytes(&b) == 0);

    /* pointers, sizes, scales */
    tlin_paged_params p = paged();
    const size_t need = tlin_paged_workspace_bytes(&p);
    CHECK(tlin_paged_attn(&p, fake, fake, fake, fake, fake, fake, fake, NULL, fake, need - 1, NULL) == TLIN_ERR_WORKSPACE);
    CHECK(tlin_paged_attn(&p, fake, fake, fake, fake, fake, fake, fake, NULL, NULL, need, NULL) == TLIN_ERR_WORKSPACE);
    CHECK(tlin_paged_attn(NULL, fake, fake, fake, fake, fake, fake, fake, NULL, fake, need, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_paged_append(NULL, NULL, NULL, NULL, fake, fake, fake, fake, fake, fake, fake, NULL, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_paged_append(&p, NULL, fake, fake, fake, fake, fake, fake, fake, fake, fake, NULL, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_rope(NULL, fake, fake, fake, (double *)fake, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_pages_copy(NULL, fake, fake, fake, NULL, 1, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_pages_reserve(NULL, fake, fake, fake, fake, fake, fake, fake, fake, much, NULL) == TLIN_ERR_INVALID_ARG);
    CHECK(tlin_pages_compact(NULL, fake, fake, fake, fake, fake, fake, fake, much, NULL) == TLIN_ERR_INVALID_ARG);
    const float scales[] = {0.f, -1.f, NAN, INFINITY};
    for (int i = 0; i < 4; ++i) {
        p.scale = scales[i];
        CHECK(tlin_paged_attn(&p, fake, fake, fake, fake, fake, fake, fake, NULL, fake, much, NULL) == TLIN_ERR_INVALID_ARG);
    }
    b.num_pages = 9; b.table_width = 3; b.S = 2;
    CHECK(tlin_pages_free(&b, fake, fake, fake, NULL, 0, NULL) == TLIN_OK);
    CHECK(tlin_pages_fork(&b, fake, fake, fake, NULL, NULL, 0, NULL, NULL) == TLIN_OK);
    CHECK(tlin_pages_reserve(&b, fake, fake, fake, fake, fake, fake, fake, (char *)fake + 16, much, NULL) == TLIN_ERR_WORKSPACE);
    b.table_stride = 2;
    CHECK(tlin_pages_workspace_bytes(&b) == 0);

    /* frequencies: every place written is inside rot / 2 */
    for (int rot = 2; rot <= 128; rot += 2)
        for (int scaling = 0; scaling < 4; ++scaling) {
            const tlin_status st = tlin_rope_frequencies(rot, 10000.0, scaling, 4.0, 4096.0, 1.0, 32.0, f, &amplitude);
            CHECK(st == (scaling == TLIN_ROPE_BASE && rot < 4 ? TLIN_ERR_INVALID_ARG : TLIN_OK));
            if (st == TLIN_OK) for (int i = 0; i < rot / 2; ++i) CHECK(isfinite(f[i]) && f[i] > 0);
        }
    CHECK(tlin_rope_frequencies(130, 10000.0, 0, 1.0, 0.0, 0.0, 0.0, f, NULL) == TLIN_ERR_INVALID_ARG);
    if (fails) return 1;
    printf("paged api driver ok\n");
    return 0;
}
