/*
 * The calls around a feature network's step and its serving, of the built
 * library, when the host has no memory left
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
    svm_packed P{reinterpret_cast<void*>((uintptr_t)6 << 20), 12, 5, 4, 32,
                 SVM_F32};
    int64_t bytes;
    float f[4];
    svm_grad g{};
    g.n = 5;  // no data
    svm_adamw_params p{1e-3, 0.9, 0.999, 1e-8, 0, 1, 1, 32};
    svm_adamw_tensor t{};
    t.n = 5;  // no memory
    check("svm_grad_norm", [&] {
        return svm_grad_norm(&g, 1, 1.0, 1.0, f, f + 1, nullptr, 0, 0,
                             nullptr);
    });
    check("svm_grad_norm_workspace",
          [&] { return svm_grad_norm_workspace(&g, 1, &bytes); });
    check("svm_adamw_step_clipped",
          [&] { return svm_adamw_step_clipped(&t, 1, &p, f, 0, nullptr); });
    check("svm_group_norm", [&] {
        return svm_group_norm(&X, 3, 2, nullptr, nullptr, 1e-5, 0, &Y, nullptr,
                              nullptr, nullptr, 0, 0, nullptr);
    });
    check("svm_group_norm_workspace", [&] {
        return svm_group_norm_workspace(6, 4, 4, 2, 0, &bytes);
    });
    check("svm_group_norm_backward", [&] {
        return svm_group_norm_backward(&X, &Y, 3, 2, f, f, nullptr, nullptr, 0,
                                       nullptr, nullptr, nullptr, nullptr,
                                       nullptr, 0, 0, nullptr);
    });
    check("svm_group_norm_backward_workspace", [&] {
        return svm_group_norm_backward_workspace(6, 3, 4, 3, 0, &bytes);
    });
    check("svm_pack_weights",
          [&] { return svm_pack_weights(&W, &P, 0, nullptr); });
    check("svm_pack_weights_bytes",
          [&] { return svm_pack_weights_bytes(5, 4, 33, 0, &bytes); });
    check("svm_unpack_weights",
          [&] { return svm_unpack_weights(&P, &W, 0, nullptr); });
    check("svm_linear_packed", [&] {
        return svm_linear_packed(&X, &P, nullptr, nullptr, 0, &Y, nullptr, 0,
                                 0, nullptr);
    });
    check("svm_linear_packed_workspace",
          [&] { return svm_linear_packed_workspace(&X, &P, &bytes); });
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
