// What the C entry points share: status and message of a refusal, the device
// check, and the guard that lets no C++ exception and no HIP error past the
// boundary.
#pragma once

#include <exception>
#include <new>
#include <string>

#include "common.hpp"

namespace msvm {

// Sets the thread's message and returns st.
svm_status fail(svm_status st, const std::string& msg);

// SVM_OK if `dev` is an ordinal of this machine's GPUs.
svm_status check_device(int dev);

// Leaves HIP's per-thread last-error slot clean on every exit, so that an
// error the library handled (or ignored while freeing) is not reported later
// by a caller's own error check.
struct ClearHipError {
    ~ClearHipError() { (void)hipGetLastError(); }
};

// Status and message of the exception at hand; nothing leaves it.  (The short
// text needs no memory of its own: it is what is told where there is none.)
inline svm_status caught() noexcept
{
    static const char* const kNoMemory = "no host memory";
    try {
        try {
            throw;
        } catch (const Error& e) {
            return fail(e.status, e.msg);
        } catch (const std::bad_alloc&) {
            return fail(SVM_E_NOMEM, kNoMemory);
        } catch (const std::exception& e) {
            return fail(SVM_E_INTERNAL, e.what());
        } catch (...) {
            return fail(SVM_E_INTERNAL, "unknown error");
        }
    } catch (...) {
        return fail(SVM_E_NOMEM, kNoMemory);
    }
}

// The thread's device is `dev` while this lives, and what it was afterwards:
// for calls that come between a caller's own device calls.  HIP's last error
// is left clean.
class OnDevice : ClearHipError {
public:
    explicit OnDevice(int dev)
    {
        HIP_TRY(hipGetDevice(&before_));
        if (before_ != dev) HIP_TRY(hipSetDevice(dev));
        else before_ = -1;
    }
    ~OnDevice()
    {
        if (before_ >= 0) (void)hipSetDevice(before_);
    }
    OnDevice(const OnDevice&) = delete;
    OnDevice& operator=(const OnDevice&) = delete;

private:
    int before_ = -1;
};

}  // namespace msvm

// Around a whole entry: no exception leaves it.  GUARD_BEGIN keeps HIP's last
// error clean too; ENTRY_BEGIN makes no HIP call by itself, so that a call that
// is refused makes none.
#define ENTRY_BEGIN try {
#define GUARD_BEGIN \
    msvm::ClearHipError clear_hip_error_on_exit_; \
    ENTRY_BEGIN
#define GUARD_END \
    } \
    catch (...) { return msvm::caught(); }
