// Host and device helpers that the operators around the pair share. Not installed.
#pragma once
#include "ficco_plan.h"

#include <initializer_list>

namespace ficco {

// A pointer argument: null where that is allowed, else device memory of the current device, aligned.
struct Arg {
    const void *ptr;
    int align;                   // bytes
    bool optional;
};

inline int check_args(std::initializer_list<Arg> args)
{
    for (const Arg &a : args) {
        if (!a.ptr && !a.optional) return FICCO_ERR_ARG;
        if ((uintptr_t)a.ptr % (uintptr_t)a.align) return FICCO_ERR_ARG;
    }
    int dev = 0;
    HIP_TRY(hipGetDevice(&dev));
    for (const Arg &a : args) {
        if (!a.ptr) continue;
        hipPointerAttribute_t at;
        if (hipPointerGetAttributes(&at, a.ptr) != hipSuccess) {
            (void)hipGetLastError();
            return FICCO_ERR_ARG;
        }
        if (at.type != hipMemoryTypeDevice || at.device != dev) return FICCO_ERR_ARG;
    }
    return FICCO_OK;
}

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Compute units of the current device; a whole MI355X where none can be asked (sizes of workspaces on a host without one).
inline int compute_units()
{
    static int of[64];
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); return 256; }
    if (dev < 64 && of[dev]) return of[dev];
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) { (void)hipGetLastError(); return 256; }
    if (dev < 64) of[dev] = cus;
    return cus;
}

// Every entry point's body: nothing leaves it as a C++ exception.
template <class Fn>
inline int guarded(Fn &&fn)
{
    try {
        return fn();
    } catch (const std::bad_alloc &) {
        return FICCO_ERR_ALLOC;
    } catch (...) {
        return FICCO_ERR_STATE;
    }
}

}  // namespace ficco
