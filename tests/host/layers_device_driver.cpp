/*
 * The host side of the feature-map calls (layers.cpp) on a machine with four
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
void linear_forward(const LinearArgs&, Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
void linear_backward(const LinearGradArgs&, Pieces& ws, hipStream_t)
{
    if (ws.run) queue();
}
void norm_forward(const NormArgs&, hipStream_t) { queue(); }
int64_t norm_backward_bytes(int64_t, int64_t) { return 0; }
void norm_backward(const NormGradArgs&, Pieces&, hipStream_t) { queue(); }
int64_t hinge_bytes(int64_t, int64_t) { return 0; }
void hinge_loss(const svm_array&, const int32_t*, float, const svm_array&,
                float*, Pieces&, hipStream_t)
{
    queue();
}
void adamw_step(const svm_adamw_tensor*, int32_t, const svm_adamw_params&,
                hipStream_t)
{
    queue();
}
void adamw_state(const int8_t*, const uint8_t*, const float*, const float*,
                 int64_t, float*, float*, hipStream_t)
{
    queue();
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
    svm_array X = arr(6, 4, 1), W = arr(5, 4, 2), Y = arr(6, 5, 3);
    svm_array dX = arr(6, 4, 4), dW = arr(5, 4, 5), N = arr(6, 4, 6);
    float f[8];
    int32_t labels[8] = {};
    int8_t m[256];
    uint8_t v[256];
    svm_adamw_params p{1e-3, 0.9, 0.999, 1e-8, 0, 1, 1, 32};
    current = 1;
    for (int turn = 0; turn < 2; ++turn) {
        broken = turn == 1;
        for (int d = 0; d < devices; ++d) {
            check("svm_linear",
                  svm_linear(&X, &W, nullptr, nullptr, 0, &Y, nullptr, nullptr,
                             0, d, nullptr),
                  d);
            check("svm_linear_backward",
                  svm_linear_backward(&Y, &X, &W, nullptr, 0, &dX, &dW,
                                      nullptr, nullptr, 0, d, nullptr),
                  d);
            check("svm_layer_norm",
                  svm_layer_norm(&X, nullptr, nullptr, 1e-5, &N, nullptr,
                                 nullptr, d, nullptr),
                  d);
            check("svm_layer_norm_backward",
                  svm_layer_norm_backward(&X, &N, f, f, nullptr, nullptr, &dX,
                                          nullptr, nullptr, nullptr, 0, d,
                                          nullptr),
                  d);
            check("svm_hinge_loss",
                  svm_hinge_loss(&X, labels, 1.0, nullptr, f, nullptr, 0, d,
                                 nullptr),
                  d);
            check("svm_adamw_step",
                  svm_adamw_step(nullptr, 0, &p, d, nullptr), d);
            check("svm_adamw_state",
                  svm_adamw_state(m, v, f, f, 4, f, f, d, nullptr), d);
        }
    }
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
