// seqmix_workspace.h -- checks and workspaces that the C entries of the token-mixing operators share (host code).
#pragma once

#include "seqmix_internal.h"

namespace cv {

#define SM_TRY(e)                       \
    do {                                \
        const int st_ = (e);            \
        if (st_ != CONV2D_OK) return st_; \
    } while (0)

constexpr int64_t kMaxRows = (1LL << 31) - 1;

inline bool known_dtype(int d) { return d == CONV2D_F32 || d == CONV2D_BF16; }
inline int64_t esize(int d) { return d == CONV2D_BF16 ? 2 : 4; }

// Rows, sequences and slots as every sequence operator has them.
inline int check_seqs(int64_t tokens, int64_t seqs, int64_t slots) {
    if (tokens < 0 || seqs < 1 || slots < 1) return CONV2D_E_INVALID;
    if (tokens > kMaxRows || seqs > kMaxRows || slots > kMaxRows) return CONV2D_E_UNSUPPORTED;
    return CONV2D_OK;
}

inline int seq_args(int64_t tokens, int64_t seqs, int64_t slots, const int64_t* off, const int32_t* slot, SeqArgs* out) {
    if (!off && tokens % seqs != 0) return CONV2D_E_INVALID;
    if (!slot && slots < seqs) return CONV2D_E_INVALID;
    *out = SeqArgs{off, slot, tokens, off ? 0 : tokens / seqs, slots, (int32_t)seqs};
    return CONV2D_OK;
}

// Rows `row` elements apart, heads `head` elements apart, of `dim` elements each, can hold what they should.
inline bool strides_ok(int64_t tokens, int64_t row, int64_t heads, int64_t head, int64_t dim) {
    if (head < dim && heads > 1) return false;
    if (head < 0 || row < 0) return false;
    // either order of rows and heads, without overlap
    const bool rows_outer = row >= (heads - 1) * head + dim;
    const bool heads_outer = heads > 1 && row >= dim && head >= (tokens - 1) * row + dim;
    return tokens <= 1 || rows_outer || heads_outer;
}

// Device memory of a descriptor, on `device`; calls that use it are ordered over streams as in conv2d.h.
struct Workspace {
    void* data = nullptr;
    int device = -1;
    hipEvent_t done = nullptr;
    hipStream_t last_stream = nullptr;
    bool has_last = false;
    // the capture that the previous captured call was part of (0: none), and its stream
    unsigned long long capture = 0;
    hipStream_t capture_stream = nullptr;

    void release() {
        if (data) (void)hipFree(data);
        if (done) (void)hipEventDestroy(done);
        data = nullptr;
        done = nullptr;
    }

    // `bytes` on the current device, once.
    int ensure(int64_t bytes) {
        if (bytes == 0) return CONV2D_OK;
        switch (alloc(bytes)) {
            case hipSuccess: return CONV2D_OK;
            case hipErrorOutOfMemory: (void)hipGetLastError(); return CONV2D_E_ALLOC;
            case hipErrorInvalidDevice: return CONV2D_E_UNSUPPORTED;
            default: return CONV2D_E_HIP;
        }
    }

    // A call waits for the previous one's workspace.  Captured calls run when their graph does: they wait for each other
    // within their graph and leave the order of the others' streams as it is.  A stream that is being captured cannot
    // be waited for from outside (its event would draw this call into the capture).
    int order_after_last(hipStream_t s) {
        if (const unsigned long long c = capture_of(s)) {
            if (capture == c && s != capture_stream) SM_TRY(wait_for(capture_stream, s));
            capture = c;
            capture_stream = s;
            return CONV2D_OK;
        }
        if (has_last && s != last_stream) {
            if (capture_of(last_stream)) return CONV2D_E_HIP;
            SM_TRY(wait_for(last_stream, s));
        }
        last_stream = s;
        has_last = true;
        return CONV2D_OK;
    }

    // Capture that stream s records into, 0: none.
    static unsigned long long capture_of(hipStream_t s) {
        hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
        unsigned long long id = 0;
        if (hipStreamGetCaptureInfo(s, &status, &id) != hipSuccess) {
            (void)hipGetLastError();
            return 0;
        }
        return status == hipStreamCaptureStatusActive ? id : 0;
    }

private:
    hipError_t alloc(int64_t bytes) {
        int dev = -1;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (device >= 0) return device == dev ? hipSuccess : hipErrorInvalidDevice;
        e = hipEventCreateWithFlags(&done, hipEventDisableTiming);
        if (e != hipSuccess) return e;
        e = hipMalloc(&data, (size_t)bytes);
        if (e != hipSuccess) {
            (void)hipEventDestroy(done);
            done = nullptr;
            data = nullptr;
            return e;
        }
        device = dev;
        return hipSuccess;
    }

    int wait_for(hipStream_t last, hipStream_t s) {
        if (hipEventRecord(done, last) != hipSuccess || hipStreamWaitEvent(s, done, 0) != hipSuccess) return CONV2D_E_HIP;
        return CONV2D_OK;
    }
};

}  // namespace cv
