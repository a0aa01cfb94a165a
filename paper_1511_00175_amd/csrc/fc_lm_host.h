// What the host sides of fc_lm.h's plans share: stream order, argument checks,
// overlap of buffers, device memory.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>
#include <new>

#include "fc_launches.h"
#include "fc_lm.h"

namespace fc {

inline int hip_code(hipError_t e) { return e == hipSuccess ? FC_OK : FC_EHIP; }

inline int dtype_bytes(int dt) { return dt == FC_F32 ? 4 : dt == FC_F16 || dt == FC_BF16 ? 2 : 0; }

// No exception leaves the C ABI.
template <typename F> int no_throw(F&& body) {
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return FC_ENOMEM;
    } catch (...) {
        return FC_EHIP;
    }
}

// Calls on one plan take effect in the order they are made: a call on another
// stream than the previous one's waits, on the device, for what is enqueued
// there.  A call enqueued while its stream is being captured runs when the
// graph is launched; it neither waits nor becomes the previous call.
struct CallOrder {
    int device = 0;
    hipStream_t last = nullptr;
    bool have_last = false;
    hipEvent_t event = nullptr;

    int create() {
        if (hipGetDevice(&device) != hipSuccess) return FC_EHIP;
        return hip_code(hipEventCreateWithFlags(&event, hipEventDisableTiming));
    }
    void destroy() {
        if (event) (void)hipEventDestroy(event);
        event = nullptr;
    }
    // Before a call enqueues anything; `note` says whether done() is due after it has.
    int begin(hipStream_t s, bool& note) {
        note = false;
        int now;
        if (hipGetDevice(&now) != hipSuccess) return FC_EHIP;
        if (now != device) return FC_EINVAL;
        if (have_last && last == s) return FC_OK;
        hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
        if (hipStreamIsCapturing(s, &st) != hipSuccess) return FC_EHIP;
        if (st != hipStreamCaptureStatusNone) return FC_OK;
        note = true;
        if (!have_last) return FC_OK;
        if (hipStreamIsCapturing(last, &st) != hipSuccess) return FC_EHIP;
        if (st != hipStreamCaptureStatusNone) return FC_EINVAL;
        if (hipEventRecord(event, last) != hipSuccess || hipStreamWaitEvent(s, event, 0) != hipSuccess) return FC_EHIP;
        return FC_OK;
    }
    void done(hipStream_t s, bool note) {
        if (!note) return;
        last = s;
        have_last = true;
    }
};

// One buffer of a call: `rows` rows of `len` elements, `ld` apart.
struct Span {
    const void* p;
    int64_t rows, len, ld;
    int bytes;     // of an element
    bool written;
    uintptr_t lo() const { return reinterpret_cast<uintptr_t>(p); }
    uintptr_t hi() const { return rows > 0 && len > 0 ? lo() + (uintptr_t)((rows - 1) * ld + len) * bytes : lo(); }
};

// Null, misaligned, badly strided or overlapping buffers.
inline int check_spans(std::initializer_list<Span> spans) {
    for (const Span& s : spans) {
        if (!s.bytes || s.rows < 0 || s.len < 0 || s.ld < s.len || s.ld >= ((int64_t)1 << 58) / (s.rows + 1)) return FC_EINVAL;
        if (s.rows > 0 && s.len > 0 && !s.p) return FC_EINVAL;
        if (s.lo() % s.bytes) return FC_EALIGN;
    }
    for (const Span* a = spans.begin(); a != spans.end(); ++a)
        for (const Span* b = a + 1; b != spans.end(); ++b)
            if ((a->written || b->written) && a->lo() < b->hi() && b->lo() < a->hi()) return FC_EALIAS;
    return FC_OK;
}

// A plan's device memory.
struct DeviceBlock {
    char* p = nullptr;
    int create(uint64_t bytes) {
        void* q = nullptr;
        if (hipMalloc(&q, bytes ? bytes : 256) != hipSuccess) {
            (void)hipGetLastError();  // the failed allocation is reported here and by no later call
            return FC_EHIP;
        }
        p = static_cast<char*>(q);
        return FC_OK;
    }
    void destroy() {
        if (p) (void)hipFree(p);
        p = nullptr;
    }
};

// Offsets of 256-byte aligned parts of a block.
struct Layout {
    uint64_t size = 0;
    uint64_t take(uint64_t bytes) {
        const uint64_t at = size;
        size += (bytes + 255) / 256 * 256;
        return at;
    }
};

}  // namespace fc
