/*
 * The AdamW step that counts the steps left out (steps.cpp) on a machine with
 * four devices that exist only here: it has to queue its work on the device
 * that it is given, and to leave the thread's own device as it was, when it
 * succeeds and when it fails.
 */
#include <cstdio>
#include <string>

#include "entry.hpp"
#include "layers.hpp"

static int current = 1, devices = 4, queued_on = -1, failures = 0;
static bool broken = false;

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
void adamw_step_counted(const svm_adamw_tensor*, int32_t,
                        const svm_adamw_params&, const float*, int64_t*,
                        hipStream_t)
{
    queued_on = current;
    if (broken) throw Error{SVM_E_DEVICE, "broken"};
}
}  // namespace msvm

int main()
{
    svm_adamw_params p{1e-3, 0.9, 0.999, 1e-8, 0, 1, 1, 32};
    float f = 1.0f;
    int64_t count = 0;
    for (int turn = 0; turn < 2; ++turn) {
        broken = turn == 1;
        for (int d = 0; d < devices; ++d) {
            const svm_status st =
                svm_adamw_step_counted(nullptr, 0, &p, &f, &count, d, nullptr);
            if (st != (broken ? SVM_E_DEVICE : SVM_OK) || queued_on != d ||
                current != 1)
                ++failures;
            current = 1;
            queued_on = -1;
        }
    }
    if (svm_adamw_step_counted(nullptr, 0, &p, &f, &count, devices, nullptr) !=
            SVM_E_INVALID ||
        queued_on != -1)
        ++failures;
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
