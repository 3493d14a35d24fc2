// Host helpers that the library's entry points share: the per-thread error
// detail, the checks of device pointers and the release of a handle's memory.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/esopt.h"

namespace es_host {

inline thread_local std::string g_last_error;

inline int fail(int code, const std::string& msg) {
    g_last_error = msg;
    return code;
}

inline int hip_fail(hipError_t e, const std::string& what) {
    return fail(ES_ERR_HIP, what + ": " + hipGetErrorString(e));
}

// A failure of call `name`: the message is formatted only here, so a call
// that succeeds builds no strings (no host allocation on its way).
inline int fail_in(int code, const char* name, const char* msg) {
    return fail(code, std::string(name) + ": " + msg);
}

inline int current_device(int* dev) {
    const hipError_t e = hipGetDevice(dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    return ES_OK;
}

// The `bytes` bytes at p must be memory that kernels on `device` can access:
// device or managed memory of that device, the whole range inside one
// allocation (checked when the runtime knows the allocation's extent), or
// mapped pinned host memory.  Catches host pointers, other devices' memory
// and overstated sizes before a kernel would fault on them.  A failed query
// leaves no error behind for later launch checks.
// (The name of the checked array is `name` followed by `part`; it is
// formatted only on failure.)
// `range`: set to the allocation that holds p, where the runtime knows it.
struct Range {
    uintptr_t base = 0;
    uint64_t size = 0;
};
inline int check_access(const void* p, uint64_t bytes, int device, const char* name,
                        const char* part, Range* range = nullptr) {
    if (bytes == 0) return ES_OK;
    auto what = [&]() { return std::string(name) + part; };
    hipPointerAttribute_t a{};
    hipError_t e = hipPointerGetAttributes(&a, p);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(ES_ERR_INVALID_ARG, what() + ": not memory the device can access");
    }
    if (a.type == hipMemoryTypeHost) {
        if (a.devicePointer == nullptr)
            return fail(ES_ERR_INVALID_ARG, what() + ": host memory not mapped for the device");
        return ES_OK;
    }
    if (a.type != hipMemoryTypeDevice && a.type != hipMemoryTypeManaged &&
        a.type != hipMemoryTypeUnified)
        return fail(ES_ERR_INVALID_ARG, what() + ": not device memory");
    if (a.type == hipMemoryTypeDevice && a.device != device)
        return fail(ES_ERR_INVALID_ARG, what() + ": memory of device " + std::to_string(a.device) +
                                            ", not of device " + std::to_string(device));
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    e = hipMemGetAddressRange(&base, &size, const_cast<void*>(p));
    if (e != hipSuccess) {                   // allocator that does not report extents
        (void)hipGetLastError();
        return ES_OK;
    }
    const uintptr_t b = reinterpret_cast<uintptr_t>(base), q = reinterpret_cast<uintptr_t>(p);
    if (q < b || q - b > size || bytes > size - (q - b))
        return fail(ES_ERR_INVALID_ARG, what() + ": " + std::to_string(bytes) +
                                            " bytes extend past the end of its allocation");
    if (range != nullptr) *range = Range{b, size};
    return ES_OK;
}

// The checks of one call's arrays: an array inside the allocation that the one
// before it was found in needs no second query (0.4 us each, and a call at a
// single token has ten arrays, most of them in one of the caller's pools).
struct Accesses {
    int device;
    const char* name;
    Range last;
    int rc = ES_OK;                         // of the first check that failed
    void check(const void* p, uint64_t bytes, const char* part) {
        if (rc != ES_OK || bytes == 0) return;
        const uintptr_t q = reinterpret_cast<uintptr_t>(p);
        if (q - last.base < last.size && bytes <= last.size - (q - last.base)) return;
        rc = check_access(p, bytes, device, name, part, &last);
    }
};

inline int check_access(const void* p, uint64_t bytes, int device, const std::string& what) {
    return check_access(p, bytes, device, what.c_str(), "");
}

// Free a plan's tile table and scratch on the plan's device: that device is made
// current for the call (the caller's is restored) and synchronised first, so
// no queued launch still reads them.  Every step runs; the first error is
// returned.
inline int release_device_memory(int device, void* tab, void* scratch, const char* name) {
    const std::string nm(name);
    int rc = ES_OK;
    int caller = -1;
    hipError_t e = hipGetDevice(&caller);
    if (e != hipSuccess) rc = hip_fail(e, nm + ": hipGetDevice");
    const bool switched = e == hipSuccess && caller != device;
    if (switched) {
        e = hipSetDevice(device);
        if (e != hipSuccess && rc == ES_OK) rc = hip_fail(e, nm + ": hipSetDevice");
    }
    e = hipDeviceSynchronize();
    if (e != hipSuccess && rc == ES_OK) rc = hip_fail(e, nm + ": hipDeviceSynchronize");
    e = hipFree(tab);
    if (e != hipSuccess && rc == ES_OK) rc = hip_fail(e, nm + ": hipFree");
    e = hipFree(scratch);
    if (e != hipSuccess && rc == ES_OK) rc = hip_fail(e, nm + ": hipFree");
    if (switched) {
        e = hipSetDevice(caller);
        if (e != hipSuccess && rc == ES_OK) rc = hip_fail(e, nm + ": hipSetDevice");
    }
    return rc;
}

}  // namespace es_host
