/*
 * The host side of the calls around a feature network's step and its serving
 * (network.cpp) on a machine with four
 * devices that exist only here: a HIP runtime of a few functions, and
 * operators that note on which device they were queued.  Every call has to
 * queue its work on the device that it is given and to leave the thread's own
 * device as it was, when it succeeds and when it fails.
 */
#include <cstdio>
#include <string>

#include "entry.hpp"
#include "layers.hpp"

static int current = 0, devices = 4, failures = 0;
static int queued_on = -1;   // device of the last operator
static bool broken = false;  // operators throw

extern "C" {
hipError_t hipGetDeviceCount(int* n) { return *n = devices, hipSuccess; }
hipError_t hipGetDevice(int* d) { return *d = current, hipSuccess; }
hipError_t hipSetDevice(int d)
{
    if (d < 0 || d >= devices) return hipErrorInvalidDevice;
    current = d;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipPeekAtLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "error"; }
}

namespace msvm {
svm_status fail(svm_status st, const std::string&) { return st; }
svm_status check_device(int dev)
{
    return dev < devices ? SVM_OK : SVM_E_INVALID;
}
static void queue()
{
    queued_on = current;
    if (broken) throw Error{SVM_E_DEVICE, "broken"};
}
void adamw_step_clipped(const svm_adamw_tensor*, int32_t,
                        const svm_adamw_params&, const float*, hipStream_t)
{
    queue();
}
void grad_norm(const svm_grad*, int32_t, double, double, float*, float*,
               Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
void group_norm(const GroupCall&, Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
void group_norm_backward(const GroupGradCall&, Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
void pack4(const svm_array&, const svm_packed&, hipStream_t) { queue(); }
void unpack4(const svm_packed&, const svm_array&, hipStream_t) { queue(); }
void linear4(const Linear4Call&, Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
}  // namespace msvm

static svm_array arr(int64_t rows, int64_t cols, uintptr_t at)
{
    return {reinterpret_cast<void*>(at << 20), rows, cols, cols, SVM_F32, 1};
}

static void check(const char* what, svm_status got, int device)
{
    const svm_status want = broken ? SVM_E_DEVICE : SVM_OK;
    if (got != want || queued_on != device || current != 1) {
        std::fprintf(stderr, "%s: status %d, queued on %d, left on %d\n", what,
                     (int)got, queued_on, current);
        ++failures;
    }
    current = 1;
    queued_on = -1;
}

int main()
{
    svm_array X = arr(6, 4, 1), Y = arr(6, 4, 2), W = arr(5, 4, 3);
    svm_array dX = arr(6, 4, 4), out = arr(6, 5, 5);
    svm_packed P{reinterpret_cast<void*>((uintptr_t)6 << 20), 1 << 20, 5, 4,
                 32, SVM_F32};
    float f[8];
    svm_grad g{f, 4, SVM_F32};
    svm_adamw_params p{1e-3, 0.9, 0.999, 1e-8, 0, 1, 1, 32};
    current = 1;
    for (int turn = 0; turn < 2; ++turn) {
        broken = turn == 1;
        for (int d = 0; d < devices; ++d) {
            check("svm_grad_norm",
                  svm_grad_norm(&g, 1, 1.0, 1.0, f, f + 1, nullptr, 0, d,
                                nullptr),
                  d);
            check("svm_adamw_step_clipped",
                  svm_adamw_step_clipped(nullptr, 0, &p, f, d, nullptr), d);
            check("svm_group_norm",
                  svm_group_norm(&X, 3, 2, nullptr, nullptr, 1e-5, 0, &Y,
                                 nullptr, nullptr, nullptr, 0, d, nullptr),
                  d);
            check("svm_group_norm_backward",
                  svm_group_norm_backward(&X, &Y, 3, 2, f, f, nullptr, nullptr,
                                          0, nullptr, &dX, nullptr, nullptr,
                                          nullptr, 0, d, nullptr),
                  d);
            check("svm_pack_weights", svm_pack_weights(&W, &P, d, nullptr), d);
            check("svm_unpack_weights", svm_unpack_weights(&P, &W, d, nullptr),
                  d);
            check("svm_linear_packed",
                  svm_linear_packed(&X, &P, nullptr, nullptr, 0, &out, nullptr,
                                    0, d, nullptr),
                  d);
        }
    }
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
