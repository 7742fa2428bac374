/*
 * The feature-map calls of the built library when the host has no memory left
 * for their messages: each has to return a status, and no exception may leave
 * a C entry.  Every call here is refused by its checks, before any device
 * call; while `none` is set, every allocation of the process fails.
 */
#include <cstdio>
#include <cstdlib>
#include <new>

#include "mi355svm.h"

static bool none = false;

void* operator new(std::size_t n)
{
    void* p = none ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

static int failures = 0;

template <class F>
static void check(const char* what, F&& call)
{
    none = true;
    const svm_status st = call();
    const char* msg = svm_last_error();
    none = false;
    if ((st != SVM_E_NOMEM && st != SVM_E_INVALID) || !msg || !msg[0]) {
        std::fprintf(stderr, "%s: status %d, message '%s'\n", what, (int)st,
                     msg ? msg : "(null)");
        ++failures;
    }
}

int main()
{
    auto arr = [](int64_t rows, int64_t cols, uintptr_t at) {
        return svm_array{reinterpret_cast<void*>(at << 20), rows, cols, cols,
                         SVM_F32, 1};
    };
    svm_array X = arr(6, 4, 1), W = arr(5, 4, 2), Y = arr(6, 7, 3);
    svm_array wrong = arr(123456, 4, 4);
    int64_t bytes;
    float f[4];
    int32_t labels[8] = {};
    svm_adamw_params p{1e-3, 0.9, 0.999, 1e-8, 0, 1, 1, 32};
    svm_adamw_tensor t{};
    t.n = 5;  // no memory
    check("svm_linear", [&] {
        return svm_linear(&X, &W, nullptr, nullptr, 0, &Y, nullptr, nullptr, 0,
                          0, nullptr);
    });
    check("svm_linear_workspace", [&] {
        return svm_linear_workspace(&X, &Y, &bytes);
    });
    check("svm_linear_backward", [&] {
        return svm_linear_backward(&Y, &X, &W, nullptr, 0, nullptr, &wrong,
                                   nullptr, nullptr, 0, 0, nullptr);
    });
    check("svm_linear_backward_workspace", [&] {
        return svm_linear_backward_workspace(&Y, &wrong, nullptr, 0, nullptr,
                                             nullptr, nullptr, &bytes);
    });
    check("svm_layer_norm", [&] {
        return svm_layer_norm(&X, nullptr, nullptr, 1e-5, &Y, nullptr, nullptr,
                              0, nullptr);
    });
    check("svm_layer_norm_backward", [&] {
        return svm_layer_norm_backward(&X, &Y, f, f, nullptr, nullptr, nullptr,
                                       nullptr, nullptr, nullptr, 0, 0,
                                       nullptr);
    });
    check("svm_layer_norm_backward_workspace", [&] {
        return svm_layer_norm_backward_workspace(-1, 4, &bytes);
    });
    check("svm_hinge_loss", [&] {
        return svm_hinge_loss(&X, labels, 1.0, &Y, f, nullptr, 0, 0, nullptr);
    });
    check("svm_hinge_loss_workspace", [&] {
        return svm_hinge_loss_workspace(6, 0, &bytes);
    });
    check("svm_adamw_step",
          [&] { return svm_adamw_step(&t, 1, &p, 0, nullptr); });
    check("svm_adamw_state", [&] {
        return svm_adamw_state(nullptr, nullptr, nullptr, nullptr, -1, f, f, 0,
                               nullptr);
    });
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
