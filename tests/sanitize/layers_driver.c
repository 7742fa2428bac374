/*
 * Drives the argument checks of the feature-map calls in a build of the
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
    svm_array X = arr(100, 40, 1 << 20), W = arr(30, 40, 1 << 21);
    svm_array Y = arr(100, 30, 1 << 22), Z = arr(100, 30, 1 << 23);
    svm_array b = arr(1, 30, 3 << 20), bad;
    int64_t bytes = -1;

    /* every type and layout through the size functions, large ones too */
    for (int t = SVM_F32; t <= SVM_F16; ++t) {
        for (int big_rows = 0; big_rows < 2; ++big_rows) {
            svm_array x = X, w = W, g = Y, dx, dw, db = b;
            x.dtype = w.dtype = g.dtype = db.dtype = t;
            if (big_rows) x.rows = g.rows = 2147483647;
            x.ld = 41;
            dx = x;
            dw = w;
            EXPECT(svm_linear_workspace(&x, &w, &bytes), SVM_OK);
            EXPECT(svm_linear_backward_workspace(&g, &x, &w, SVM_ACT_COS, &dx,
                                                 &dw, &db, &bytes),
                   SVM_OK);
            EXPECT(svm_layer_norm_backward_workspace(x.rows, 2097152, &bytes),
                   SVM_OK);
            EXPECT(svm_hinge_loss_workspace(x.rows, 2097152, &bytes), SVM_OK);
        }
    }
    EXPECT(svm_linear_workspace(NULL, &W, &bytes), SVM_E_INVALID);
    EXPECT(svm_linear_workspace(&X, &W, NULL), SVM_E_INVALID);
    bad = X;
    bad.rows = (int64_t)1 << 31;
    EXPECT(svm_linear_workspace(&bad, &W, &bytes), SVM_E_INVALID);

    /* accepted by every check but the device's */
    NO_DEVICE(svm_linear(&X, &W, &b, &Z, SVM_ACT_GELU, &Y, NULL, work, big,
                         no_gpu, NULL));
    NO_DEVICE(svm_linear(&X, &W, NULL, &Y, SVM_ACT_NONE, &Y, &Z, work, big,
                         no_gpu, NULL));
    NO_DEVICE(svm_layer_norm(&X, NULL, NULL, 1e-5, &X, NULL, NULL, no_gpu,
                             NULL));
    /* refused */
    EXPECT(svm_linear(&X, &W, &b, &Z, 99, &Y, NULL, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_linear(&X, &W, &b, &Z, SVM_ACT_GELU, &Y, &Y, work, big, no_gpu,
                      NULL),
           SVM_E_INVALID);
    EXPECT(svm_linear(&X, &W, &b, NULL, SVM_ACT_GELU, &X, NULL, work, big,
                      no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_linear(&X, &W, &b, NULL, SVM_ACT_GELU, &Y, NULL, work, big, -1,
                      NULL),
           SVM_E_INVALID);
    bad = X;
    bad.on_device = 0;
    EXPECT(svm_linear(&bad, &W, &b, NULL, SVM_ACT_GELU, &Y, NULL, work, big,
                      no_gpu, NULL),
           SVM_E_UNSUPPORTED);
    EXPECT(svm_linear_backward(&Y, &X, &W, NULL, SVM_ACT_GELU, NULL, NULL, &b,
                               work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_linear_backward(&Y, &X, &W, &Z, SVM_ACT_GELU, NULL, &W, &b,
                               work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_layer_norm(&X, &b, NULL, 1e-5, &X, NULL, NULL, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_layer_norm(&X, NULL, NULL, NAN, &X, NULL, NULL, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_layer_norm_backward(&X, &X, NULL, NULL, NULL, NULL, NULL, NULL,
                                   NULL, NULL, 0, no_gpu, NULL),
           SVM_E_INVALID);
    float f = 0;
    int32_t lab[4] = {0, 0, 0, 0};
    EXPECT(svm_hinge_loss(&X, NULL, 1.0, NULL, &f, work, big, no_gpu, NULL),
           SVM_E_INVALID);
    EXPECT(svm_hinge_loss(&X, lab, INFINITY, NULL, &f, work, big, no_gpu,
                          NULL),
           SVM_E_INVALID);

    svm_adamw_params p;
    memset(&p, 0, sizeof p);
    p.lr = 1e-3;
    p.beta1 = 0.9;
    p.beta2 = 0.999;
    p.grad_scale = 1;
    p.step = 1;
    p.bits = 8;
    svm_adamw_tensor t[3];
    memset(t, 0, sizeof t);  /* tensors of no values need no memory */
    NO_DEVICE(svm_adamw_step(t, 3, &p, no_gpu, NULL));
    NO_DEVICE(svm_adamw_step(NULL, 0, &p, no_gpu, NULL));
    t[2].n = 5;
    EXPECT(svm_adamw_step(t, 3, &p, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_adamw_step(t, -1, &p, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_adamw_step(NULL, 1, &p, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_adamw_step(t, 3, NULL, no_gpu, NULL), SVM_E_INVALID);
    p.step = 0;
    EXPECT(svm_adamw_step(t, 2, &p, no_gpu, NULL), SVM_E_INVALID);
    EXPECT(svm_adamw_state(NULL, NULL, NULL, NULL, 4, &f, NULL, no_gpu, NULL),
           SVM_E_INVALID);

    if (failures) {
        fprintf(stderr, "%d checks failed\n", failures);
        return 1;
    }
    puts("all checks passed");
    return 0;
}
