/* Host-side checks of the calls around a reduced activation, built against a
 * copy of the library whose host code is compiled with AddressSanitizer: the
 * argument structures and the pointer array are heap blocks of exactly their
 * size, so a read past one is reported.  Every call either fails validation or,
 * with valid-looking arguments, fails at its launch because no GPU is visible;
 * the program refuses to run when one is, since its pointers are not real device
 * memory. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "xred.h"

static int failures = 0;

#define EXPECT(call, want)                                                                \
    do {                                                                                  \
        xred_status got_ = (call);                                                        \
        if (got_ != (want)) {                                                             \
            fprintf(stderr, "line %d: %s returned %d (%s), expected %d: %s\n", __LINE__, #call, \
                    (int)got_, xred_status_string(got_), (int)(want), xred_last_error());  \
            ++failures;                                                                   \
        }                                                                                 \
    } while (0)

/* a made-up device address, 4 GiB from the others */
static void *fake(uintptr_t k) { return (void *)(uintptr_t)(0x7f0000000000ull + (k << 32)); }

static xred_rows rows(uintptr_t k, uint64_t stride)
{
    xred_rows r = {fake(k), stride};
    return r;
}

/* a heap copy of exactly the structure */
static void *heap(const void *args, size_t size)
{
    void *p = malloc(size);
    memcpy(p, args, size);
    return p;
}

#define CALL(name, args, want)                              \
    do {                                                    \
        void *h_ = heap(&(args), sizeof(args));             \
        EXPECT(name(h_, NULL), want);                       \
        free(h_);                                           \
    } while (0)

static const xred_dtype types[3] = {XRED_FLOAT32, XRED_BFLOAT16, XRED_FLOAT16};

int main(void)
{
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) == hipSuccess && ndev > 0) {
        printf("skipped: a GPU is visible\n");
        return 0;
    }
    const xred_status NODEV = XRED_HIP_ERROR;

    /* xred_fold_norm: every count of sources, every shape of rows */
    EXPECT(xred_fold_norm(NULL, NULL), XRED_INVALID_ARGUMENT);
    static const uint64_t hiddens[] = {1, 7, 64, 130, 512, 513, 4096, 8200, 16390, 32768};
    for (unsigned t = 0; t < 3; ++t)
        for (unsigned h = 0; h < sizeof hiddens / sizeof *hiddens; ++h)
            for (uint32_t n = 1; n <= XRED_MAX_SRC; n = n < 5 ? n + 1 : 2 * n > 64 && n < 64 ? 64 : 2 * n) {
                const void **srcs = malloc(sizeof(void *) * n);
                for (uint32_t i = 0; i < n; ++i) srcs[i] = fake(100 + i);
                xred_fold_norm_args a = {0};
                a.srcs = srcs;
                a.src_stride = hiddens[h];
                a.nsrc = n;
                a.rows = 3;
                a.hidden = hiddens[h];
                a.out = rows(1, hiddens[h]);
                a.sum = rows(2, hiddens[h] + 3);
                a.out8 = rows(3, hiddens[h]);
                a.group = 512;
                a.scale = rows(4, (hiddens[h] + 511) / 512);
                a.weight = fake(5);
                a.rstd = fake(6);
                a.dtype = types[t];
                a.weight_dtype = n % 2 ? types[t] : XRED_FLOAT32;
                a.eps = 1e-6f;
                CALL(xred_fold_norm, a, NODEV);
                a.residual = rows(7, hiddens[h]);
                a.rstd = fake(7);
                CALL(xred_fold_norm, a, XRED_ALIAS);
                a.rstd = NULL;
                a.srcs = NULL;
                CALL(xred_fold_norm, a, XRED_INVALID_ARGUMENT);
                a.rows = 0;      /* no sources are looked at */
                CALL(xred_fold_norm, a, XRED_SUCCESS);
                a.nsrc = 65;
                CALL(xred_fold_norm, a, XRED_INVALID_ARGUMENT);
                free(srcs);
            }

    /* xred_fold_norm_grad */
    EXPECT(xred_fold_norm_grad(NULL, NULL), XRED_INVALID_ARGUMENT);
    for (unsigned t = 0; t < 3; ++t)
        for (unsigned h = 0; h < sizeof hiddens / sizeof *hiddens; ++h) {
            xred_fold_norm_grad_args a = {0};
            a.rows = 1000;
            a.hidden = hiddens[h];
            a.dout = rows(1, hiddens[h]);
            a.sum = rows(2, hiddens[h]);
            a.dsum = rows(3, hiddens[h]);
            a.dx = a.dsum;
            a.weight = fake(4);
            a.rstd = fake(5);
            a.dweight = fake(6);
            a.workspace = fake(7);
            a.workspace_bytes = xred_fold_norm_grad_workspace(1000, hiddens[h]);
            a.dtype = types[t];
            a.weight_dtype = types[t];
            CALL(xred_fold_norm_grad, a, NODEV);
            --a.workspace_bytes;
            CALL(xred_fold_norm_grad, a, XRED_INVALID_ARGUMENT);
            a.dweight = NULL;
            a.workspace = NULL;
            a.workspace_bytes = 0;
            CALL(xred_fold_norm_grad, a, NODEV);
            a.rows = 0;
            CALL(xred_fold_norm_grad, a, XRED_SUCCESS);
        }

    /* xred_route and xred_route_grad */
    EXPECT(xred_route(NULL, NULL), XRED_INVALID_ARGUMENT);
    EXPECT(xred_route_grad(NULL, NULL), XRED_INVALID_ARGUMENT);
    static const uint32_t experts[] = {1, 16, 60, 128, 200, 256, 500, 1024};
    for (unsigned t = 0; t < 3; ++t)
        for (unsigned e = 0; e < sizeof experts / sizeof *experts; ++e)
            for (int score = 0; score < 2; ++score) {
                xred_route_args a = {0};
                a.tokens = 5000;
                a.experts = experts[e];
                a.topk = experts[e] < 8 ? experts[e] : 8;
                a.groups = experts[e] % 4 ? 1 : 4;
                a.group_topk = 1;
                a.group_score = 2;
                a.flags = XRED_ROUTE_RENORM;
                a.logits = rows(1, experts[e]);
                a.bias = fake(2);
                a.ids = fake(3);
                a.weights = fake(4);
                a.dtype = types[t];
                a.score = (xred_score)score;
                a.scale = 1.0f;
                CALL(xred_route, a, NODEV);
                a.weights = (float *)(void *)a.ids;
                CALL(xred_route, a, XRED_ALIAS);
                a.groups = experts[e] + 1;
                CALL(xred_route, a, XRED_INVALID_ARGUMENT);
                xred_route_grad_args b = {0};
                b.tokens = 5000;
                b.experts = experts[e];
                b.topk = a.topk;
                b.logits = rows(1, experts[e]);
                b.dlogits = rows(2, experts[e]);
                b.ids = fake(3);
                b.dweights = fake(4);
                b.dtype = types[t];
                b.score = (xred_score)score;
                b.scale = 1.0f;
                CALL(xred_route_grad, b, NODEV);
                b.dlogits = b.logits;
                CALL(xred_route_grad, b, XRED_ALIAS);
            }

    /* xred_dispatch_plan, with and without a workspace */
    EXPECT(xred_dispatch_plan(NULL, NULL), XRED_INVALID_ARGUMENT);
    static const uint64_t tokens[] = {0, 1, 512, 513, 100000, INT32_MAX / 8};
    for (unsigned n = 0; n < sizeof tokens / sizeof *tokens; ++n) {
        xred_dispatch_plan_args a = {0};
        a.tokens = tokens[n];
        a.experts = 1024;
        a.topk = 8;
        a.ids = fake(1);
        a.counts = fake(100);
        a.offsets = fake(101);
        a.pos = fake(40);
        a.slots = n % 2 ? fake(80) : NULL;
        a.workspace_bytes = xred_dispatch_plan_workspace(8 * tokens[n], 1024);
        a.workspace = a.workspace_bytes ? fake(102) : NULL;
        CALL(xred_dispatch_plan, a, NODEV);
        if (a.workspace_bytes) {
            --a.workspace_bytes;
            CALL(xred_dispatch_plan, a, XRED_INVALID_ARGUMENT);
        }
        a.counts = NULL;
        CALL(xred_dispatch_plan, a, XRED_INVALID_ARGUMENT);
    }

    /* xred_dispatch, xred_combine and xred_combine_grad */
    EXPECT(xred_dispatch(NULL, NULL), XRED_INVALID_ARGUMENT);
    EXPECT(xred_combine(NULL, NULL), XRED_INVALID_ARGUMENT);
    EXPECT(xred_combine_grad(NULL, NULL), XRED_INVALID_ARGUMENT);
    for (int t = XRED_FLOAT32; t <= XRED_UINT8; ++t)
        for (unsigned h = 0; h < sizeof hiddens / sizeof *hiddens; ++h)
            for (uint32_t k = 1; k <= XRED_MAX_TOPK; k = k < 3 ? k + 1 : k + 7) {
                const uint64_t n = hiddens[h];
                xred_dispatch_args a = {0};
                a.tokens = 1000;
                a.hidden = n;
                a.out_rows = 900;
                a.scale_columns = 2;
                a.topk = k;
                a.dtype = (xred_dtype)t;
                a.x = rows(1, n);
                a.out = rows(2, n + 1);
                a.scale = rows(3, 2);
                a.out_scale = rows(4, 2);
                a.pos = fake(5);
                CALL(xred_dispatch, a, NODEV);
                a.out_scale = a.scale;
                CALL(xred_dispatch, a, XRED_ALIAS);
                a.out_scale.data = NULL;
                CALL(xred_dispatch, a, XRED_INVALID_ARGUMENT);
                const int row_type = t == XRED_FLOAT32 || t == XRED_BFLOAT16 || t == XRED_FLOAT16;
                xred_combine_args b = {0};
                b.tokens = 1000;
                b.hidden = n;
                b.y_rows = 900;
                b.topk = k;
                b.dtype = (xred_dtype)t;
                b.y = rows(1, n);
                b.base = rows(2, n);
                b.out = b.base;
                b.pos = fake(3);
                b.weights = fake(4);
                CALL(xred_combine, b, row_type ? NODEV : XRED_UNSUPPORTED);
                b.out = b.y;
                CALL(xred_combine, b, row_type ? XRED_ALIAS : XRED_UNSUPPORTED);
                xred_combine_grad_args c = {0};
                c.tokens = 1000;
                c.hidden = n;
                c.y_rows = 900;
                c.topk = k;
                c.dtype = (xred_dtype)t;
                c.dout = rows(1, n);
                c.y = rows(2, n);
                c.dy = c.y;
                c.pos = fake(3);
                c.weights = fake(4);
                c.dweights = fake(5);
                CALL(xred_combine_grad, c, row_type ? NODEV : XRED_UNSUPPORTED);
                c.dy = c.dout;
                CALL(xred_combine_grad, c, row_type ? XRED_ALIAS : XRED_UNSUPPORTED);
            }

    if (failures == 0) printf("all layer checks passed\n");
    return failures ? 1 : 0;
}
