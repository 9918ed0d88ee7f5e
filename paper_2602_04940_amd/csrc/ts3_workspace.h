// A device buffer of an object that grows when a call needs more of it.  Included by ts3.hip after
// its error helpers.
#pragma once

namespace {

// Whether `st` is being captured into a graph.  A stream that cannot tell counts as captured.
bool stream_captures(hipStream_t st) {
    hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &s) == hipSuccess) return s != hipStreamCaptureStatusNone;
    (void)hipGetLastError();
    return true;
}

ts3_status device_alloc(void **p, int64_t bytes) {
    hipError_t e = hipMalloc(p, (size_t)bytes);
    if (e == hipSuccess) return TS3_OK;
    (void)hipGetLastError();
    *p = nullptr;
    return fail(e == hipErrorOutOfMemory ? TS3_ERR_OUT_OF_MEMORY : TS3_ERR_HIP, "hipMalloc(%lld bytes): %s",
                (long long)bytes, hipGetErrorString(e));
}

// A captured graph holds the buffer's address, and its replays use it whenever they come: a buffer
// that a capture has seen is kept until the owner goes, one that none has seen is freed when it is
// replaced.  Nothing is allocated inside a capture.
struct Workspace {
    void *p = nullptr;
    int64_t bytes = 0;
    bool captured = false;
    std::vector<void *> kept;

    // At least `need` bytes for a call on `st`; `total`, the owner's device bytes, follows.
    ts3_status reserve(int64_t need, hipStream_t st, int64_t &total) {
        const bool capturing = stream_captures(st);
        if (need <= bytes) {
            captured = captured || (capturing && p);
            return TS3_OK;
        }
        if (capturing)
            return fail(TS3_ERR_BAD_STATE, "a workspace of %lld bytes has to be allocated, which a stream capture does not "
                        "allow: make the call once before it", (long long)need);
        HIP_TRY(hipDeviceSynchronize());
        if (captured) {
            try {
                kept.push_back(p);
            } catch (const std::bad_alloc &) {
                return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
            }
        } else {
            (void)hipFree(p);
            total -= bytes;
        }
        p = nullptr;
        bytes = 0;
        captured = false;
        ts3_status s = device_alloc(&p, need);
        if (s != TS3_OK) return s;
        bytes = need;
        total += need;
        return TS3_OK;
    }
    void free() {
        (void)hipFree(p);
        for (void *q : kept) (void)hipFree(q);
        p = nullptr;
        kept.clear();
    }
};

}  // namespace
