// Host-side checks that the entry points of the 8-bit integer layers share.
#pragma once

#include "../../include/shadowtutor.h"
#include "st_internal.h"

namespace st {

constexpr int64_t kMaxInt8Extent = 0x7fffffff;      // rows, channels
constexpr int kMaxInt8K = 131071;                   // (-128)^2 of each fits a 32-bit sum
constexpr int64_t kMaxInt8N = 4194240;              // 65535 tiles of 64 channels, a grid's second extent

// whether [rows][cols] at these strides spans at most 2^48 elements (extents are at most kMaxInt8Extent)
inline bool extent_fits(int64_t rows, int64_t row_stride, int64_t cols, int64_t col_stride)
{
    return (double)rows * (double)row_stride + (double)cols * (double)col_stride <= 281474976710656.0;
}

// `rows` pieces of `width` bytes, `pitch` apart
struct Pieces {
    uintptr_t begin; int64_t rows, width, pitch;
    uintptr_t end() const { return begin + (uintptr_t)((rows - 1) * pitch + width); }
};
// Whether two matrices may share a byte.  Rows of one that lie between the rows of the other (columns of one buffer) do not; of matrices of different pitches
// only the extents are looked at.
inline bool may_share(Pieces a, Pieces b)
{
    if (a.end() <= b.begin || b.end() <= a.begin) return false;
    for (Pieces* p : {&a, &b})
        if (p->rows > 1 && p->pitch < p->width) *p = {p->begin, 1, (int64_t)(p->end() - p->begin), 0};
    if ((a.rows == 1 && b.rows == 1) || (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch)) return true;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch, between = (int64_t)(b.begin - a.begin) % pitch, at = between < 0 ? between + pitch : between;
    return at < a.width || at + b.width > pitch;
}

// The buffers of a call: device memory of the current device, aligned to their elements, none that is written sharing a byte with another.
// The first fault is kept as the thread's error text.
class Int8Buffers {
public:
    explicit Int8Buffers(const char* call) : call_(call)
    {
        if (cudaGetDevice(&device_) != cudaSuccess) { cudaGetLastError(); status_ = fail_on_thread(ST_ERR_CUDA, "%s: no current device", call); }
    }
    int device() const { return device_; }
    bool ok() const { return status_ == ST_OK; }
    st_status status() const { return (st_status)status_; }
    void add(const char* name, const void* q, int64_t element, int64_t count, bool written) { add(name, q, element, 1, count, 0, written); }
    void add(const char* name, const void* q, int64_t element, int64_t rows, int64_t columns, int64_t pitch, bool written)
    {
        if (!ok()) return;
        const Pieces p = {(uintptr_t)q, rows, columns * element, pitch * element};
        cudaPointerAttributes at;
        const char* fault = nullptr;
        if (!q) fault = "is NULL";
        else if (p.begin % element) fault = "is not aligned to its elements";
        else if (cudaPointerGetAttributes(&at, q) != cudaSuccess) { cudaGetLastError(); fault = "is not memory of the current device"; }
        else if (at.type != cudaMemoryTypeManaged && !(at.type == cudaMemoryTypeDevice && at.device == device_)) fault = "is not memory of the current device";
        for (int i = 0; i < n_ && !fault; ++i)
            if ((written || seen_[i].written) && may_share(p, seen_[i].p)) fault = "overlaps another buffer of the call";
        if (fault) { status_ = fail_on_thread(ST_ERR_INVALID_ARG, "%s: %s %s", call_, name, fault); return; }
        seen_[n_++] = {p, written};
    }

private:
    struct Seen { Pieces p; bool written; } seen_[8];
    const char* call_;
    int device_ = 0, n_ = 0, status_ = ST_OK;
};

}  // namespace st
