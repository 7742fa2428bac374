/*
 * Drives the argument checks and the plans of the calls around a feature
 * network's step and its serving in a build of the
 * library whose host code carries AddressSanitizer and
 * UndefinedBehaviorSanitizer (a CPU test: every call here is refused before
 * any device work, by the checks or because there is no device; no pointer
 * into device memory is followed).  Exits 0 when every call returned the
 * expected status with a message.
 */
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "mi355svm.h"

static int failures = 0;

static void expect(svm_status got, svm_status want, int line)
{
    const char* msg = svm_last_error();
    if (got != want) {
        fprintf(stderr, "line %d: status %d, expected %d (%s)\n", line,
                (int)got, (int)want, msg ? msg : "(null)");
        ++failures;
    } else if (want != SVM_OK && (!msg || !msg[0])) {
        fprintf(stderr, "line %d: no error message\n", line);
        ++failures;
    }
}
#define EXPECT(call, want) expect((call), (want), __LINE__)

/* no device, or (on a machine that has one) an ordinal past the last */
static void expect_no_device(svm_status got, int line)
{
    if (got != SVM_E_DEVICE && got != SVM_E_INVALID) {
        fprintf(stderr, "line %d: status %d, expected a refusal\n", line,
                (int)got);
        ++failures;
    }
}
#define NO_DEVICE(call) expect_no_device((call), __LINE__)

static svm_array arr(int64_t rows, int64_t cols, uintptr_t at)
{
    svm_array a;
    memset(&a, 0, sizeof a);
    a.data = (void*)at;
    a.rows = rows;
    a.cols = cols;
    a.ld = cols;
    a.dtype = SVM_F32;
    a.on_device = 1;
    return a;
}

int main(void)
{
    const int64_t big = (int64_t)1 << 60;
    void* work = (void*)(uintptr_t)(1 << 24);
    const int no_gpu = 1 << 20;
    svm_array X = arr(100, 40, 1 << 20), Y = arr(100, 40, 1 << 21);
    svm_array W = arr(30, 40, 1 << 22), O = arr(100, 30, 1 << 23), bad;
    svm_packed P = {(void*)(uintptr_t)(1 << 26), big, 30, 40, 64, SVM_F32};
    int64_t bytes = -1;
    float f[2] = {0, 0};

    /* every type through the size functions, the smallest and the largest */
    static const int64_t sizes[][4] = {
        {0, 1, 1, 1},          {1, 1, 1, 1},
        {2147483647, 1, 2097152, 2097152},
        {2147483647, 2147483647, 2097152, 1},
        {2147483647, 1, 8, 1}, {2147483646, 2, 2097152, 4096},
        {6, 3, 24, 3},         {1 << 20, 1 << 20, 30, 6},
        {1 << 20, 1 << 10, 231, 33}};
    for (int t = SVM_F32; t <= SVM_F16; ++t) {
        for (size_t i = 0; i < sizeof sizes / sizeof *sizes; ++i) {
            const int64_t* s = sizes[i];
            EXPECT(svm_group_norm_workspace(s[0], s[1], s[2], s[3], t, &bytes),
                   SVM_OK);
            EXPECT(svm_group_norm_backward_workspace(s[0], s[1], s[2], s[3], t,
                                                     &bytes),
                   SVM_OK);
        }
        EXPECT(svm_pack_weights_bytes(2097152, 2097152, 32, t, &bytes),
               SVM_OK);
        for (int many = 0; many < 2; ++many) {
            svm_array x = X;
            svm_packed w = P;
            x.dtype = w.dtype = t;
            x.rows = many ? 2147483647 : 1;
            x.ld = 41;
            EXPECT(svm_linear_packed_workspace(&x, &w, &bytes), SVM_OK);
        }
    }
    svm_grad g[300];
    for (int i = 0; i < 300; ++i) {
        g[i].data = (void*)(uintptr_t)((1 << 20) + 16 * i);
        g[i].n = i % 7 ? i : (int64_t)1 << 40;
        g[i].dtype = i % 3;
    }
    EXPECT(svm_grad_norm_workspace(g, 300, &bytes), SVM_OK);

    /* accepted by every check but the device's */
    NO_DEVICE(svm_grad_norm(g, 300, 1.0, 1.0, f, f + 1, work, big, no_gpu,
                            NULL));
    NO_DEVICE(svm_grad_norm(NULL, 0, 1.0, INFINITY, f, NULL, NULL, 0, no_gpu,
                            NULL));
    NO_DEVICE(svm_group_norm(&X, 25, 4, NULL, NULL, 1e-5, SVM_ACT_SILU, &X,
                             NULL, NULL, work, big, no_gpu, NULL));
    bad = X;
    bad.ld = (int64_t)1 << 40;  /* rows far apart */
    NO_DEVICE(svm_group_norm(&bad, 25, 4, NULL, NULL, 1e-5, SVM_ACT_SILU, &Y,
                             NULL, NULL, work, big, no_gpu, NULL));
    NO_DEVICE(svm_group_norm_backward(&X, &Y, 25, 4, f, f, NULL, NULL,
                                      SVM_ACT_RELU, NULL, &X, NULL, NULL, work,
                                      big, no_gpu, NULL));
    NO_DEVICE(svm_pack_weights(&W, &P, no_gpu, NULL));
    NO_DEVICE(svm_unpack_weights(&P, &W, no_gpu, NULL));
    NO_DEVICE(svm_linear_packed(&X, &P, NULL, &O, SVM_ACT_GELU, &O, work, big,
                                no_gpu, NULL));
    /* refused */
    EXPECT(svm_grad_norm(g, -1, 1.0, 1.0, f, NULL, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_grad_norm(NULL, 1, 1.0, 1.0, f, NULL, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_grad_norm(g, 300, 1.0, NAN, f, NULL, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_group_norm(&X, 7, 4, NULL, NULL, 1e-5, 0, &Y, NULL, NULL, work,
                          big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_group_norm(&X, 25, 3, NULL, NULL, 1e-5, 0, &Y, NULL, NULL, work,
                          big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_group_norm(&X, 25, 4, NULL, NULL, 1e-5, 0, NULL, NULL, NULL,
                          work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_group_norm_backward(&X, NULL, 25, 4, f, f, NULL, NULL, 0, NULL,
                                   &Y, NULL, NULL, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    P.group = 48;
    EXPECT(svm_pack_weights(&W, &P, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_linear_packed_workspace(&X, &P, &bytes), SVM_E_INVALID);
    P.group = 64;
    P.bytes = 100;
    EXPECT(svm_unpack_weights(&P, &W, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_linear_packed(&X, &P, NULL, NULL, 0, &O, work, big, no_gpu,
                             NULL),
           SVM_E_INVALID);
    svm_adamw_params p;
    memset(&p, 0, sizeof p);
    EXPECT(svm_adamw_step_clipped(NULL, 0, &p, f, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_adamw_step_clipped(NULL, 0, NULL, f, no_gpu, NULL),
           SVM_E_INVALID);

    if (failures) {
        fprintf(stderr, "%d checks failed\n", failures);
        return 1;
    }
    puts("all checks passed");
    return 0;
}
