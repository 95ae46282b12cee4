// Argument checks that several C entry points share (host code).
#pragma once

#include "logits.cuh"

namespace sr {

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Whether all of these (NULL or not) lie on the boundary of a 32-bit number.
template <typename... P>
inline bool aligned_4(const P*... p) { return (aligned(p, 4) && ...); }

inline bool short_of(const void* ws, size_t have, size_t need) { return ws == nullptr || have < need || !aligned(ws, 16); }

constexpr double kLargest = 3.4028234663852886e38;   // what fp32 holds
constexpr int64_t kMaxPitch = int64_t(1) << 31;      // rows * pitch * 4 bytes stay below 2^64

// Rows of `width` elements that are written: they are those that are read themselves, or none of them meets one of those.
inline int check_rows(const void* in, int64_t pitch, const void* out, int64_t out_pitch, int32_t dtype, int32_t n_rows, int32_t width) {
    if (out_pitch < width || out_pitch > kMaxPitch) return SR_ERR_BAD_SIZE;
    if (n_rows == 0) return SR_OK;
    if (out == nullptr) return SR_ERR_NULL;
    const int64_t size = dtype_bytes(dtype);
    if (!aligned(out, (size_t)size)) return SR_ERR_ALIGN;
    const uint64_t a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(out);
    const auto bytes = [&](int64_t row) { return ((uint64_t)(n_rows - 1) * (uint64_t)row + (uint64_t)width) * (uint64_t)size; };       // below 2^64
    const uint64_t a_end = a + bytes(pitch), b_end = b + bytes(out_pitch);
    if (a_end <= b || b_end <= a) return SR_OK;
    if (pitch != out_pitch) return n_rows == 1 && a == b ? SR_OK : SR_ERR_OVERLAP;
    const int64_t off = ((((int64_t)(b - a)) / size) % pitch + pitch) % pitch;              // column of the one in a row of the other
    return a == b || (off >= width && off + width <= pitch) ? SR_OK : SR_ERR_OVERLAP;
}

}  // namespace sr
