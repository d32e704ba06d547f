// What the entry points of the operators check alike, and how they walk over sequences.
#pragma once
#include <algorithm>
#include <cstdint>
#include <string>
#include <vector>

#include "operators.h"
#include "status.h"

namespace lfmmi {
namespace {

constexpr int64_t kCacheBytes = (int64_t)256 << 20;  // behind the L2s

inline size_t dtype_size(int32_t dtype) { return dtype == LFMMI_F32 ? 4 : 2; }

inline bool known(int32_t dtype) { return dtype == LFMMI_F32 || dtype == LFMMI_BF16 || dtype == LFMMI_F16; }

inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

inline lfmmi_status check_lengths(const int32_t* lengths, int32_t B, int32_t T)
{
    if (lengths)
        for (int32_t b = 0; b < B; ++b)
            if (lengths[b] < 0 || lengths[b] > T)
                return fail(LFMMI_ERR_INVALID_ARG, "lengths[" + std::to_string(b) + "] outside [0, T]");
    return LFMMI_OK;
}

// Strides of rows (b, t); no offset passes 64 bits.
inline lfmmi_status check_strides(int64_t stride_b, int64_t stride_t, int32_t B, int32_t T)
{
    if (stride_b < 0 || stride_t < 0) return fail(LFMMI_ERR_INVALID_ARG, "strides must be >= 0");
    if (stride_b > ((int64_t)1 << 60) / std::max(B, 1) || stride_t > ((int64_t)1 << 60) / std::max(T, 1))
        return fail(LFMMI_ERR_UNSUPPORTED, "strides beyond 2^60 elements");
    return LFMMI_OK;
}

// Sequences that one launch takes, and their lengths.
inline int32_t fill_lengths(const int32_t* lengths, int32_t b, int32_t B, SeqLengths* out)
{
    if (!lengths) {
        out->n = 0;
        return B - b;
    }
    const int32_t n = std::min(B - b, kLengthsPerLaunch);
    out->n = n;
    std::copy(lengths + b, lengths + b + n, out->T);
    return n;
}

template <typename U>
inline U* at(U* p, int64_t i)
{
    return p ? p + i : nullptr;
}

inline const void* at_bytes(const void* p, int64_t i)
{
    return p ? static_cast<const char*>(p) + i : nullptr;
}
inline void* at_bytes(void* p, int64_t i) { return p ? static_cast<char*>(p) + i : nullptr; }

struct Span {
    uintptr_t at, end;
    bool written;
};

// Whether an array that is written overlaps another array.
inline bool overlap(std::vector<Span>& spans)
{
    const auto before = [](const Span& a, const Span& b) { return a.at < b.at; };
    if (!std::is_sorted(spans.begin(), spans.end(), before))
        std::sort(spans.begin(), spans.end(), before);
    uintptr_t any = 0, written = 0;  // ends of what came before
    for (const Span& s : spans) {
        if (s.at < written || (s.written && s.at < any)) return true;
        any = std::max(any, s.end);
        if (s.written) written = std::max(written, s.end);
    }
    return false;
}

}  // namespace
}  // namespace lfmmi
