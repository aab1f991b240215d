// sf_host.hpp -- what the entry points' host code shares: errors, the checks of
// pointers and strides, kernel timing, the device's size.
#pragma once
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <string>
#include <utility>
#include <vector>

#include <hip/hip_runtime.h>

#include "stateflow.h"

#define TRY(x)                          \
    do {                                \
        sf_status _rc = (x);            \
        if (_rc != SF_OK) return _rc;   \
    } while (0)

namespace sf {
namespace host {

// the last failure of the calling thread (sf_last_error)
inline thread_local std::string g_err;

inline sf_status fail(sf_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return s;
}

inline sf_status hip_fail(hipError_t e, const char *what) {
    return fail(SF_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

struct Dim {
    int64_t size, stride;
};

// Strided tensor with a contiguous innermost dim of `inner` elements: the index
// map is injective iff, sorted by stride, each stride covers the previous extent.
inline bool non_overlapping(std::vector<Dim> dims, int64_t inner) {
    std::vector<Dim> d;
    for (auto &x : dims)
        if (x.size > 1) d.push_back(x);
    std::sort(d.begin(), d.end(), [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t extent = inner;
    for (auto &x : d) {
        if (x.stride < extent) return false;
        extent = x.stride * x.size;
    }
    return true;
}

// byte extent of a tensor, as integer addresses ([lo, hi); lo = 0 for an
// absent tensor): no pointer arithmetic on absent (NULL) pointers and no
// ordering of pointers into different objects
struct Range {
    uintptr_t lo, hi;
    const char *name;
};
inline Range span(const void *p, int64_t bytes, const char *name) {
    const uintptr_t b = (uintptr_t)p;
    return {b, b && bytes > 0 ? b + (uintptr_t)bytes : b, name};
}
inline Range wsrange(const void *ws, size_t bytes) { return span(ws, (int64_t)bytes, "ws"); }
inline bool overlap(const Range &a, const Range &b) {
    return a.lo && b.lo && a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi;
}
inline sf_status check_alias(const std::vector<Range> &ins, const std::vector<Range> &outs) {
    for (size_t i = 0; i < outs.size(); ++i) {
        for (auto &in : ins)
            if (overlap(outs[i], in)) return fail(SF_E_ALIAS, "output %s overlaps input %s", outs[i].name, in.name);
        for (size_t j = i + 1; j < outs.size(); ++j)
            if (overlap(outs[i], outs[j]))
                return fail(SF_E_ALIAS, "output %s overlaps output %s", outs[i].name, outs[j].name);
    }
    return SF_OK;
}
inline sf_status check_align(std::initializer_list<std::pair<const void *, const char *>> ps) {
    for (auto &p : ps)
        if (p.first && ((uintptr_t)p.first % 16))
            return fail(SF_E_ALIGN, "%s is not 16-byte aligned", p.second);
    return SF_OK;
}

constexpr size_t ALIGN = 256;
inline size_t al(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }

// Compute units of the current device (256 on MI355X; also the fallback when no
// device is visible, e.g. for workspace queries on a host without a GPU).
inline int device_cus() {
    static thread_local int cached_dev = -2, cached_cus = 256;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev != cached_dev) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
            (void)hipGetLastError();
            n = 256;
        }
        cached_dev = dev;
        cached_cus = n;
    }
    return cached_cus;
}

inline sf_status check_timing(const sf_tuning *t) {
    if (t && (t->overlap < 0 || t->overlap > 2))
        return fail(SF_E_SHAPE, "tuning.overlap must be 0, 1 or 2 (got %d)", t->overlap);
    const sf_timing *tm = t ? t->timing : nullptr;
    if (!tm) return SF_OK;
    if (tm->capacity < 0 || tm->count < 0 || tm->count > tm->capacity)
        return fail(SF_E_SHAPE, "timing: need 0 <= count <= capacity (count=%d capacity=%d)", tm->count,
                    tm->capacity);
    if (tm->capacity > 0 && (!tm->start || !tm->stop || !tm->kind))
        return fail(SF_E_NULL, "timing: start, stop and kind arrays are required");
    return SF_OK;
}
inline sf_timing *timing_of(const sf_tuning *t) { return t ? t->timing : nullptr; }

inline void take_pair(sf_timing *tm, int kind, hipEvent_t &e0, hipEvent_t &e1) {
    e0 = e1 = nullptr;
    if (!tm || kind < 0 || kind >= 32 || !((tm->mask >> kind) & 1u)) return;
    if (tm->count >= tm->capacity) {
        ++tm->dropped;
        return;
    }
    e0 = (hipEvent_t)tm->start[tm->count];
    e1 = (hipEvent_t)tm->stop[tm->count];
    tm->kind[tm->count] = kind;
    ++tm->count;
}

}  // namespace host
}  // namespace sf
