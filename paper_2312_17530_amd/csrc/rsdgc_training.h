// What the training operators (rsdgc_norm.hip, rsdgc_head.hip) share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/rsdgc.h"

namespace rsdgc {

// Keeps `what` and the error for rsdgc_last_hip_error(); returns RSDGC_EHIP (rsdgc_kernels.hip).
int remember_hip_error(hipError_t e, const char *what);

inline bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline size_t type_size(int32_t dtype) { return dtype == RSDGC_BF16 ? 2 : 4; }
inline bool type_known(int32_t dtype) { return dtype == RSDGC_F32 || dtype == RSDGC_BF16; }

// Bytes that rows x cols elements with a row stride of ld take.
inline size_t extent_bytes(int64_t rows, int64_t cols, int64_t ld, size_t size) {
    return rows <= 0 ? 0 : (static_cast<size_t>(rows - 1) * static_cast<size_t>(ld) + static_cast<size_t>(cols)) * size;
}
inline bool ranges_overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && x < y + nb && y < x + na;
}

// What an operand takes in memory; of a matrix also the bytes from row to row and of a row.
struct Range {
    const void *p;
    size_t n, pitch, row;
};
inline Range matrix_range(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t size) {
    return {p, extent_bytes(rows, cols, ld, size), static_cast<size_t>(ld) * size, static_cast<size_t>(cols) * size};
}
// Columns of one buffer side by side do not overlap, though one begins before the other ends.
inline bool ranges_overlap(const Range &a, const Range &b) {
    if (!ranges_overlap(a.p, a.n, b.p, b.n)) return false;
    if (!a.pitch || a.pitch != b.pitch) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const size_t off = y >= x ? (y - x) % a.pitch : (a.pitch - (x - y) % a.pitch) % a.pitch;       // of b's rows behind a's
    return off < a.row || off + b.row > a.pitch;
}

typedef __bf16 bf16;

template <typename T> __device__ __forceinline__ float to_float(T v) { return static_cast<float>(v); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

}  // namespace rsdgc
