// The vocabulary head under a loss, in pieces of the vocabulary: softmax cross entropy against one target per token, and
// distillation from a teacher's top logits (gfx950, wave64).
//
//   z[n][v] = x_n . W_v / t             lse_n = log sum_v exp z[n][v]
//   loss_n  = t^2 sum_v q[n][v] (log q[n][v] - (z[n][v] - lse_n))      q: the answer, a distribution over few v
//   d[n][v] = t g_n (exp(z[n][v] - lse_n) - q[n][v])                   g_n: gradient of the token's loss
//   dx = d W,  dW = d^T x
// Cross entropy is the case t = 1, q = 1 at the target.  The logits are never kept: the forward pass leaves a maximum and a sum
// of exponentials per token and strip of the vocabulary, the backward pass forms d for one piece of the vocabulary at a time
// and takes both products of it.
//
// Planes.  The matrix instructions take 16-bit operands and add in float32.  What has to count as float32 is held as several
// 16-bit planes whose sum it is; the product of two such operands is the sum of the products of those planes that matter.
//   many rows  float16, hi = f16(s a) and lo = f16(s a - hi), with a power of two s that brings the largest magnitude to
//              2^14 .. 2^15: 22 bits of every element down to 2^-17 of the largest, below that an absolute error of 2^-40 of it.
//              Three products (lo*lo is under 2^-22 of hi*hi), and a pass over the operand to find s.
//              "Largest" is of a row for x under the logits, of a piece for W, of a token for d.  A token's gain g = m 2^e goes
//              apart: d has m, dx's row 2^e at the end, and x under dW 2^e beforehand, with one scale over the rows; so no token
//              knows how large another's gradient or x is, but for the sum over tokens, dW.
//                float32   x, W and d as two planes
//                bfloat16  logits from x and W as they are; dW from d as two planes and x as one (its 8 bits fit), because dW
//                          goes to a float32 arena; dx from d as two planes and W as one.  dx is bfloat16 itself, yet 11 bits of
//                          d are not enough: a token's d sums up to nothing, so that what W's rows have in common leaves dx but
//                          for the roundings of d (a shared part a hundred times the rest: dx 2e-2 off with 11 bits, 1.7e-3, its
//                          own rounding, with 22)
//   few rows   bfloat16, three planes of 8 bits each, which keep float32's range and need no scale.  Six products for two
//              operands of three planes; x and W in bfloat16 are taken as they are.  More products, but these are hidden behind
//              the reading of W, and W is not gone over beforehand: float32 W is split on its way from memory to registers.
//
// What it measured (all of a forward and backward pass; W's rows by width by tokens):
//   131072 x 4096 x 8192 bfloat16   stats 6.7 to 7.1 ms = 1.24 to 1.32 PFLOP/s, d 7.2 (1.23), dx 13.9 of two products (1.27), dW 12.5 of
//                                   two products (1.40); a large library product on this card reaches 1.44.  Bound by the matrix
//                                   instructions' rate under the card's power (busy 60 to 84 % of the cycles); d loses to its epilogue,
//                                   4 bytes of planes for each logit
//   32000 x 1024 x 2048 float32     383 + 406 + 350 + 356 us, three products each: 1.1 PFLOP/s of 16-bit products, 360 TFLOP/s of
//                                   float32 ones, where the float32 matrix instructions reach 150
//   65536 x 4096 x 1 bfloat16       104 us for 537 MB: 5.2 TB/s, bound by memory
#include "rsdgc_gemm.h"
#include "rsdgc_training.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

namespace rsdgc {
namespace {

using namespace gemm;

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kMaxParts = 1024;                    // workgroups of a search for the largest magnitude
constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxVocab = int64_t(1) << 26, kMaxStride = int64_t(1) << 20;
constexpr int64_t kRowChunk = 16384;               // rows that are taken through the backward pass together
constexpr int64_t kRowChunkForward = 65536;        // ... through the forward pass
constexpr int64_t kPieceBytes = int64_t(512) << 20;   // d's planes of one piece of the vocabulary
constexpr int64_t kMaxPiece = int64_t(1) << 24;       // its rows: those of a tile of 64, beyond the last as well, lie within 2^31 bytes of d
constexpr int64_t kPackBytes = int64_t(256) << 20;    // a piece of W laid out as planes
constexpr int64_t kPackBytesRare = int64_t(64) << 20; // the same where only an unaligned W needs it

// Scales are powers of two, kept as exponents: those of x under the products of dW, of a piece of W.
enum Shift { kShiftX, kShiftW, kShifts = 16 };
constexpr int kTop = 14;                           // the exponent that a scale brings the largest magnitude to: 2^14 .. 2^15
constexpr float kNoExponent = -10000.0f;           // of nothing

// Up to so many rows a call takes the form for few rows.  Measured, few / many, us, W of 32768 rows (as is: both read as they lie):
//   loss alone                     with gradients
//   float32   x 4096  384 rows: 556 / 710, 512: 704 / 732, 768: 1036 / 876     128 rows: 957 / 1465, 192: 1533 / 1605, 256: 1760 / 1664
//   float32   x 515   384 rows: 84 / 90, 512: 110 / 96                         128 rows: 198 / 200, 192: 250 / 242
//   bfloat16  x 4097  384 rows: 187 / 323, 1024: 430 / 445, 2048: 829 / 684    192 rows: 951 / 1298, 256: 1220 / 1365, 333: 1566 / 1504
//   bfloat16  x 4096, as is: the same                                          128 rows: 539 / 633, 160: 757 / 703, 192: 809 / 727
int64_t few_rows(int32_t dtype, bool as_is, bool backward) {
    const bool unaligned = dtype == RSDGC_BF16 && !as_is;
    return backward ? (unaligned ? 256 : 160) : unaligned ? 1024 : 384;
}
// ------------------------------------------------------------------ answers
// A token's answer: `top` entries idx / q (q NULL: ones), an entry counts where 0 <= idx < vocab.
struct Answers {
    const int32_t *idx;
    const float *q;
    int32_t top;
    int32_t vocab;
};

// The teacher's entries of the rows.
struct Teacher {
    const int32_t *idx;
    const float *logit;
    int32_t top, vocab;
    float inv_t;
};
// Distillation: q of a row's entries from the teacher's logits, entries that name the same token merged into the first of them.
// By one wave; `room`: 2 * top words of LDS of its own.  Returns whether the row has an answer.
__device__ __forceinline__ bool row_answers(const Teacher &a, int64_t row, int32_t *room, int32_t *idx, float *q) {
    const int lane = threadIdx.x & 63, top = a.top;
    int32_t *at = room;
    float *e = reinterpret_cast<float *>(room + top);
    float most = -INFINITY;
    for (int k = lane; k < top; k += 64) {
        const int32_t i = a.idx[row * top + k];
        const float l = a.logit[row * top + k];
        const bool counts = i >= 0 && i < a.vocab && l > -INFINITY;     // NaN: no
        at[k] = counts ? i : -1;
        e[k] = l;
        if (counts) most = fmaxf(most, l);
    }
    most = wave_max(most);
    float sum = 0.0f;
    for (int k = lane; k < top; k += 64) {
        // a teacher that is certain (an infinite logit) splits its certainty among those; the temperature comes after the difference, so
        // that float32's lowest and largest values stay what they are
        e[k] = at[k] < 0 ? 0.0f : most == INFINITY ? (e[k] == INFINITY ? 1.0f : 0.0f) : exp2f((e[k] - most) * a.inv_t * kLog2e);
        sum += e[k];
    }
    sum = wave_sum(sum);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");              // the other lanes' entries
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    for (int k = lane; k < top; k += 64) {
        const int32_t i = at[k];
        bool first = i >= 0, again = false;
#pragma unroll 8
        for (int j = 0; j < top; ++j) {
            first &= at[j] != i || j >= k;
            again |= at[j] == i && j > k;
        }
        float s = e[k];
        if (first && again)                                             // rare
            for (int j = k + 1; j < top; ++j) s += at[j] == i ? e[j] : 0.0f;
        idx[k] = first ? i : -1;
        q[k] = first ? s * inv : 0.0f;
    }
    return sum > 0.0f;
}
// The same for all rows, a wave each, and the backward pass's gain: t * g_n, +0 for a row without an answer.
__global__ __launch_bounds__(256) void k_answers(const Teacher a, int64_t rows, int32_t *idx, float *q, const float *row_grad, float t, float *gain) {
    extern __shared__ int32_t lds_answers[];       // [4][2][top]
    const int wave = threadIdx.x >> 6;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + wave; row < rows; row += static_cast<int64_t>(gridDim.x) * 4) {
        const bool any = row_answers(a, row, lds_answers + wave * 2 * a.top, idx + row * a.top, q + row * a.top);
        if ((threadIdx.x & 63) == 0) gain[row] = any ? t * row_grad[row] : 0.0f;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // the room has been read
    }
}

// ------------------------------------------------------------------- planes
__device__ __forceinline__ float finite_magnitude(float v) {
    const float m = fabsf(v);
    return m < INFINITY ? m : 0.0f;
}
// |v| = m * 2^e with 1 <= m < 2; 0 for zero, infinities and NaN.
__device__ __forceinline__ int exponent_of(float v) { return v != 0.0f && fabsf(v) < INFINITY ? ilogbf(v) : 0; }
// The same of the largest of several magnitudes, as a float; kNoExponent for 0.
__device__ __forceinline__ float exponent_of_most(float most) { return most > 0.0f ? static_cast<float>(ilogbf(most)) : kNoExponent; }
// The exponent of the scale that brings magnitudes up to 2^most to kTop.
__device__ __forceinline__ int shift_for(float most) { return most > kNoExponent ? kTop - static_cast<int>(most) : 0; }
// A token's gain as it counts in d of many rows, with an exponent of its own: d then has all its bits whatever the other tokens' gains are,
// and the rest of the gain, 2^(exponent_of(gain) - kTop), is taken up by dx's row and by x under dW.
__device__ __forceinline__ float gain_in_d(float gain) { return ldexpf(gain, kTop - exponent_of(gain)); }
__device__ __forceinline__ float block_max(float v, float *red) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < static_cast<int>(blockDim.x >> 6); ++w) v = fmaxf(v, red[w]);
    return v;
}

// Eight elements of a row at c, zeros beyond its end: 16-byte loads at any alignment of the elements.
template <typename T>
__device__ __forceinline__ void load_chunk(const T *row, int c, int cols, float (&to)[8]) {
    if (c + 8 <= cols) {
        T q[8];
        __builtin_memcpy(q, row + c, sizeof(q));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = to_float(q[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = c + e < cols ? to_float(row[c + e]) : 0.0f;
    }
}

// The exponent of the largest finite magnitude of a matrix; a partial result per workgroup.  Bound by memory: 16384 x 4096 bfloat16, a piece of W,
// 41 us = 3.3 TB/s (16 bytes a thread, no atomics: a search's order must not matter).
template <typename T>
__global__ __launch_bounds__(256) void k_largest(const T *x, int64_t rows, int32_t cols, int64_t ld, float *parts) {
    __shared__ float red[4];
    float most = 0.0f;
    const int chunks = (cols + 7) / 8;
    // a workgroup goes over the chunks of all rows, 8 elements a thread
    int64_t r = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / chunks;
    int c = static_cast<int>((static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) % chunks);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    const int64_t down = stride / chunks;
    const int along = static_cast<int>(stride % chunks);
    while (r < rows) {
        float v[8];
        load_chunk(x + r * ld, 8 * c, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_magnitude(v[e]));
        r += down;
        c += along;
        if (c >= chunks) { c -= chunks; ++r; }
    }
    most = block_max(most, red);
    if (threadIdx.x == 0) parts[blockIdx.x] = exponent_of_most(most);
}

// t * g_n of the rows: from an array, or (one target a row, t = 1) as they are needed.
struct Gains {
    const float *gain, *row_grad;
    const int32_t *target;
    int32_t vocab;
    __device__ __forceinline__ float of(int64_t n) const {
        if (gain) return gain[n];
        const int32_t i = target[n];
        return i >= 0 && i < vocab ? row_grad[n] : 0.0f;
    }
};

template <typename H>
__device__ __forceinline__ void split(float v, H &hi, H &lo) {
    hi = static_cast<H>(v);
    const float rest = v - static_cast<float>(hi);
    lo = static_cast<H>(fabsf(static_cast<float>(hi)) < INFINITY ? rest : 0.0f);     // infinities and NaN stay in hi
}
__device__ __forceinline__ uint16_t bits(_Float16 v) { return __builtin_bit_cast(uint16_t, v); }
__device__ __forceinline__ uint16_t bits(bf16 v) { return __builtin_bit_cast(uint16_t, v); }

// A matrix as float16 planes under the scale that `parts` gives (hi, and lo where it is wanted), rows of `ld_out` (a multiple
// of 8) elements, zeros beyond cols.  gain not NULL: each row times the power of two of its gain, zeros where the gain is 0.
// Bound by memory: 16384 x 4096 bfloat16 to one plane 43 us = 6.3 TB/s, its reads still in the cache from the search before.
template <typename T>
__global__ __launch_bounds__(256) void k_planes(const T *x, int64_t rows, int32_t cols, int64_t ld, const float *gain, const float *parts, int32_t n_parts,
                                                int32_t *shift_out, uint16_t *hi, uint16_t *lo, int32_t ld_out) {
    __shared__ float red[4];
    float most = kNoExponent;
    for (int i = threadIdx.x; i < n_parts; i += 256) most = fmaxf(most, parts[i]);
    const int shift = shift_for(block_max(most, red));
    if (blockIdx.x == 0 && threadIdx.x == 0) *shift_out = shift;
    const int chunks = ld_out / 8;
    int64_t r = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / chunks;
    int c = static_cast<int>((static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) % chunks);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    const int64_t down = stride / chunks;
    const int along = static_cast<int>(stride % chunks);
    while (r < rows) {
        float v[8];
        load_chunk(x + r * ld, 8 * c, cols, v);
        const float g = gain ? gain[r] : 1.0f;
        const int by = shift + exponent_of(g);
        uint16_t h8[8], l8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(g != 0.0f ? ldexpf(v[e], by) : 0.0f, h, l);
            h8[e] = bits(h);
            l8[e] = bits(l);
        }
        *reinterpret_cast<uint4 *>(hi + r * ld_out + 8 * c) = *reinterpret_cast<const uint4 *>(h8);
        if (lo) *reinterpret_cast<uint4 *>(lo + r * ld_out + 8 * c) = *reinterpret_cast<const uint4 *>(l8);
        r += down;
        c += along;
        if (c >= chunks) { c -= chunks; ++r; }
    }
}

// By a workgroup: a thread's part of a row's largest finite magnitude, and the row as planes under a scale of its own.
template <typename T>
__device__ __forceinline__ float largest_of_row(const T *x, int cols) {
    float most = 0.0f;
    for (int c = threadIdx.x * 8; c < cols; c += 256 * 8) {
        float v[8];
        load_chunk(x, c, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_magnitude(v[e]));
    }
    return most;
}
template <typename T>
__device__ __forceinline__ void row_as_planes(const T *x, int cols, int shift, int32_t *shift_out, uint16_t *hi, uint16_t *lo, int ld_out) {
    if (threadIdx.x == 0) *shift_out = shift;
    for (int c = threadIdx.x * 8; c < ld_out; c += 256 * 8) {
        float v[8];
        load_chunk(x, c, cols, v);
        uint16_t h8[8], l8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(ldexpf(v[e], shift), h, l);
            h8[e] = bits(h);
            l8[e] = bits(l);
        }
        *reinterpret_cast<uint4 *>(hi + c) = *reinterpret_cast<const uint4 *>(h8);
        *reinterpret_cast<uint4 *>(lo + c) = *reinterpret_cast<const uint4 *>(l8);
    }
}
// x of the logits, with a scale for each row: none coarsens the others.
__global__ __launch_bounds__(256) void k_planes_by_row(const float *x, int32_t cols, int64_t ld, int32_t *shift_out, uint16_t *hi, uint16_t *lo, int32_t ld_out) {
    __shared__ float red[4];
    const int64_t r = blockIdx.x;
    const float most = block_max(largest_of_row(x + r * ld, cols), red);
    row_as_planes(x + r * ld, cols, shift_for(exponent_of_most(most)), shift_out + r, hi + r * ld_out, lo + r * ld_out, ld_out);
}

// The backward pass's gain of each row, t * g_n, +0 for rows without an answer (whatever g_n holds there), and the exponent of the largest
// finite magnitude of gain times x.  float32: x's rows that have a gain as planes, under a scale for each (see k_planes_by_row).
template <typename T>
__global__ __launch_bounds__(256) void k_gain(const Answers a, const float *row_grad, float t, const T *x, int64_t rows, int32_t cols, int64_t ld, float *gain, float *parts, int32_t *shift_out,
                                              uint16_t *hi, uint16_t *lo, int32_t ld_out) {
    __shared__ float red[4];
    float most = kNoExponent;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        bool mine = false;
        for (int k = threadIdx.x; k < a.top; k += 256) {
            const int32_t i = a.idx[r * a.top + k];
            mine |= i >= 0 && i < a.vocab;
        }
        const bool any = __syncthreads_or(mine);
        const float g = any ? t * row_grad[r] : 0.0f;
        if (threadIdx.x == 0) gain[r] = g;
        if (g == 0.0f) continue;
        float most_x = exponent_of_most(block_max(largest_of_row(x + r * ld, cols), red));
        if (sizeof(T) == 4) row_as_planes(x + r * ld, cols, shift_for(most_x), shift_out + r, hi + r * ld_out, lo + r * ld_out, ld_out);
        if (most_x > kNoExponent) most = fmaxf(most, most_x + static_cast<float>(exponent_of(g)));
    }
    if (threadIdx.x == 0) parts[blockIdx.x] = most;
}

// Three bfloat16 planes whose sum is v.
__device__ __forceinline__ void split3(float v, uint16_t (&p)[3]) {
    bf16 h = static_cast<bf16>(v);
    if (!(fabsf(to_float(h)) < INFINITY) && fabsf(v) < INFINITY) h = __builtin_bit_cast(bf16, static_cast<uint16_t>(__builtin_bit_cast(uint32_t, v) >> 16));   // rounded beyond the range
    const bool in = fabsf(to_float(h)) < INFINITY;       // infinities and NaN stay in the first plane
    const float rest = in ? v - to_float(h) : 0.0f;
    const bf16 m = static_cast<bf16>(rest), l = static_cast<bf16>(rest - to_float(m));
    p[0] = bits(h);
    p[1] = bits(m);
    p[2] = bits(l);
}

// Matrices as bfloat16 planes (float32: three, bfloat16: a copy), rows of ld_out (a multiple of 8) elements, zeros beyond cols
// and in rows whose gain is 0.
template <typename T>
struct Plain {
    const T *x;
    int64_t rows, ld;
    uint16_t *out;
    int64_t plane;
    Gains gains;
    int masked;                        // by the gains
    int out_only;                      // all zeros
};
template <typename T>
__device__ __forceinline__ void lay_plain(const Plain<T> &m, int cols, int ld_out, int64_t first, int64_t stride) {
    constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
    const int chunks = ld_out / 8;
    int64_t r = first / chunks;
    int c = static_cast<int>(first % chunks);
    const int64_t down = stride / chunks;
    const int along = static_cast<int>(stride % chunks);
    while (r < m.rows) {
        float v[8];
        load_chunk(m.x + r * m.ld, 8 * c, cols, v);
        const bool in = !m.out_only && (!m.masked || m.gains.of(r) != 0.0f);
        uint16_t o[3][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint16_t p[3];
            split3(in ? v[e] : 0.0f, p);
#pragma unroll
            for (int q = 0; q < kPlanes; ++q) o[q][e] = p[q];
        }
#pragma unroll
        for (int q = 0; q < kPlanes; ++q) *reinterpret_cast<uint4 *>(m.out + q * m.plane + r * ld_out + 8 * c) = *reinterpret_cast<const uint4 *>(o[q]);
        r += down;
        c += along;
        if (c >= chunks) { c -= chunks; ++r; }
    }
}
// Few rows: x.
template <typename T>
__global__ __launch_bounds__(256) void k_plain(const Plain<T> a, int32_t cols, int32_t ld_out) {
    lay_plain<T>(a, cols, ld_out, static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, static_cast<int64_t>(gridDim.x) * 256);
}
// The same behind a teacher: a row for each wave, its answer and gain before.
template <typename T>
__global__ __launch_bounds__(256) void k_plain_taught(const Plain<T> a, int32_t cols, int32_t ld_out, const Teacher teacher, int32_t *idx, float *q, const float *row_grad, float t,
                                                      float *gain) {
    extern __shared__ int32_t lds_answers[];       // [4][2][top]
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    if (row >= a.rows) return;
    const bool any = row_answers(teacher, row, lds_answers + wave * 2 * teacher.top, idx + row * teacher.top, q + row * teacher.top);
    const float g = any ? t * row_grad[row] : 0.0f;
    if (lane == 0) gain[row] = g;
    Plain<T> mine = a;                             // this row alone, in or out
    mine.x += row * a.ld;
    mine.out += row * ld_out;
    mine.rows = 1;
    mine.gains = {nullptr, nullptr, nullptr, 0};
    mine.masked = 0;
    if (g == 0.0f) mine.out_only = 1;
    lay_plain<T>(mine, cols, ld_out, lane, 64);
}

// Rows that the loads to LDS cannot take as they are: copied to rows of a multiple of 8 elements.
__global__ __launch_bounds__(256) void k_align(const bf16 *x, int64_t rows, int32_t cols, int64_t ld, uint16_t *out, int32_t ld_out) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x * 8; c < ld_out; c += 256 * 8) {
            uint16_t q[8];
            if (c + 8 <= cols) __builtin_memcpy(q, x + r * ld + c, sizeof(q));
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = c + e < cols ? bits(x[r * ld + c + e]) : 0;
            *reinterpret_cast<uint4 *>(out + r * ld_out + c) = *reinterpret_cast<const uint4 *>(q);
        }
}

__global__ __launch_bounds__(256) void k_clear(float *p, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) p[i] = 0.0f;
}

// ------------------------------------------------------------------ forward
// C[v][n]: a lane has one token and 16 rows of the vocabulary per block, so that a strip's maximum and sum of exponentials are
// formed in registers and one exchange between the wave's halves; 8 bytes for each token and strip are all that is written.
// One target a row: its logit, which is left out of the strips, so that the loss of a token that is nearly sure of its answer, the
// logarithm of 1 + little, is as good as the little.
// A teacher's entries: their logits, of the same sums as the strips', so that what is wrong with them cancels in a small loss.
struct Picked {
    const int32_t *target;             // one token a row, or NULL
    const int32_t *entries;            // ... or `top` of them
    int32_t top;
    float *logit;                      // [n][max(1, top)]
    int32_t first;                     // vocabulary row that the piece begins with
};
// The logits of those entries of tokens n0 .. n0 + count that name one of `rows` vocabulary rows from `from` on; at(token, row) is in LDS.
template <int THREADS, typename F>
__device__ __forceinline__ void pick(const Picked &p, int n0, int count, int from, int rows, const F &at) {
    const int32_t *entries = p.entries + static_cast<int64_t>(n0) * p.top;
    float *logit = p.logit + static_cast<int64_t>(n0) * p.top;
    const int all = count * p.top;
#pragma unroll 4
    for (int i = 4 * threadIdx.x; i < all; i += 4 * THREADS) {
        int32_t four[4] = {-1, -1, -1, -1};
        if (i + 4 <= all) __builtin_memcpy(four, entries + i, sizeof(four));
        else
#pragma unroll
            for (int u = 0; u < 4; ++u) four[u] = i + u < all ? entries[i + u] : -1;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t v = static_cast<uint32_t>(four[u]) - static_cast<uint32_t>(from);     // negative entries: beyond
            if (v < static_cast<uint32_t>(rows)) logit[i + u] = at((i + u) / p.top, static_cast<int>(v));
        }
    }
}
struct StatsArgs {
    const int32_t *shift_x, *shift_w;  // of scaled planes, by row and of the piece; NULL: none
    float inv_t;
    float2 *stats;                     // [n][strips]: maximum, sum of exponentials around it
    int32_t strips, first_strip;       // strip of the piece's first row
    Picked picked;
};
template <class S>
__global__ __launch_bounds__(S::kThreads, 2) void k_stats(const Problem p, const StatsArgs e) {
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    int tm, tn, part;
    tile_of(p, blockIdx.x, tm, tn, part);
    typename S::Sums acc;
    product<S>(p, tm, tn, part, (lds_char *)lds, acc);
    const Place<S> at(tm, tn);
    const int shift_w = e.shift_w ? *e.shift_w : 0;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int n = at.col(j);
        const float unit = ldexpf(e.inv_t, -shift_w - (n < p.n && e.shift_x ? e.shift_x[n] : 0));
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                acc[i][j][r] = at.row(i, r) < p.m ? acc[i][j][r] * unit : -INFINITY;
                most = fmaxf(most, acc[i][j][r]);
            }
        if (e.picked.target) {
            const int32_t target = n < p.n ? e.picked.target[n] : -1, from = e.picked.first + at.row0;
            if (target >= from && target < e.picked.first + min(p.m, at.row0 + S::MI * 32)) {       // rare
                const int own = target - from - 4 * (at.lane >> 5);                // one of the wave's halves has it
                float logit = 0.0f;
                most = -INFINITY;
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool it = 32 * i + 8 * (r >> 2) + (r & 3) == own;
                        logit = it ? acc[i][j][r] : logit;
                        acc[i][j][r] = it ? -INFINITY : acc[i][j][r];
                        most = fmaxf(most, acc[i][j][r]);
                    }
                if (((target - from) >> 2 & 1) == at.lane >> 5) e.picked.logit[n] = logit;
            }
        }
        most = fmaxf(most, __shfl_xor(most, 32));
        const float around = most > -INFINITY ? most : 0.0f;     // nothing but -inf, or nothing in the vocabulary: a sum of 0
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - around) * kLog2e);
        sum += __shfl_xor(sum, 32);
        if (at.lane < 32 && n < p.n && at.row0 < p.m) e.stats[static_cast<int64_t>(n) * e.strips + e.first_strip + at.row0 / (S::MI * 32)] = make_float2(most, sum);
    }
    if (!e.picked.entries) return;
    // the tile's logits through LDS, those of one strip after the other: [token][row]
    constexpr int kDown = S::MI * 32, kLine = kDown + 4;
    static_assert(S::TN * kLine * 4 <= S::kLds, "room for a strip");
    float *tile = reinterpret_cast<float *>(lds);
    for (int strip = 0; strip < S::WM; ++strip) {
        __syncthreads();                           // the last stage, or the strip before, has been read
        if (static_cast<int>(threadIdx.x >> 6) / S::WN == strip)
#pragma unroll
            for (int j = 0; j < S::NI; ++j)
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *reinterpret_cast<float4 *>(tile + (at.col(j) - tn * S::TN) * kLine + 32 * i + 2 * r + 4 * (at.lane >> 5)) =
                            make_float4(acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]);
        __syncthreads();
        const int v0 = tm * S::TM + strip * kDown;
        pick<S::kThreads>(e.picked, tn * S::TN, min(S::TN, p.n - tn * S::TN), e.picked.first + v0, max(0, min(kDown, p.m - v0)),
                          [&](int n, int v) { return tile[n * kLine + v]; });
    }
}

// lse from a token's strips, and the loss, a wave for each token.  picked: the logits of its one target (see Picked), or of a teacher's
// entries, whose shares are formed here.  4096 tokens: 7 us for a target, 13 behind 64 entries.  To hand 64 entries a token on costs k_stats
// 12 % (65536 x 2048 x 4096 bfloat16 979 / 1097 us), dot products with W's rows here cost 164 us.
template <bool TAUGHT>
__global__ __launch_bounds__(256) void k_loss(int64_t rows, const float2 *stats, int32_t strips, const int32_t *target, const float *picked, int32_t vocab, const Teacher teacher, float t,
                                              float *loss, float *lse_out) {
    extern __shared__ int32_t lds_answers[];       // [4][4][top]: idx, q, and room
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    if (row >= rows) return;
    const float2 *s = stats + row * strips;
    // a running maximum and sum, eight strips at a time
    float most = -INFINITY, sum = 0.0f;
    for (int c = lane; c < strips; c += 64 * 8) {
        float2 q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = c + 64 * u < strips ? s[c + 64 * u] : make_float2(-INFINITY, 0.0f);
        float m = most;
#pragma unroll
        for (int u = 0; u < 8; ++u) m = fmaxf(m, q[u].x);
        const float around = m > -INFINITY ? m : 0.0f;
        sum *= exp2f((most - around) * kLog2e);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += q[u].y * exp2f((q[u].x - around) * kLog2e);
        most = m;
    }
    const float all = wave_max(most), around = all > -INFINITY ? all : 0.0f;
    sum *= exp2f((most - around) * kLog2e);
    sum = wave_sum(sum);
    if constexpr (!TAUGHT) {
        const int32_t i = target[row];
        if (lane) return;
        if (i < 0 || i >= vocab) {
            loss[row] = 0.0f;
            lse_out[row] = around + logf(sum);
        } else {
            const float z = picked[row], top = fmaxf(all, z);
            const float others = sum == 0.0f ? 0.0f : sum * exp2f((around - top) * kLog2e), own = exp2f((z - top) * kLog2e);
            loss[row] = z >= all ? log1pf(others) : (top - z) + logf(others + own);
            lse_out[row] = top + logf(others + own);
        }
        return;
    }
    const int top = teacher.top;
    int32_t *idx = lds_answers + wave * 4 * top;
    float *q = reinterpret_cast<float *>(idx + top);
    row_answers(teacher, row, idx + 2 * top, idx, q);
    const float log_sum = logf(sum);
    float l = 0.0f;
    for (int k = lane; k < top; k += 64)                          // a lane's own entries
        if (idx[k] >= 0 && q[k] > 0.0f) l += q[k] * (logf(q[k]) + ((around - picked[row * top + k]) + log_sum));
    l = wave_sum(l);
    if (lane) return;
    loss[row] = t * (t * l);                       // the square may leave the range
    lse_out[row] = around + log_sum;
}

// ----------------------------------------------------------------- backward
// C[n][v]: d as planes.  PAIRED: two neighbouring columns a lane, so that a store takes 4 bytes.  A piece of
// d takes kPieceBytes at most (two passes of 131072 x 4096 x 8192: 43.3 ms with 128 MB, 41.0 with 256, 40.6 with 512).
struct GradArgs {
    int many;                          // many rows: d has the gain's fraction alone (gain_in_d)
    const int32_t *shift_x, *shift_w;  // of scaled planes that the logits come from, by row and of the piece; NULL: none
    float inv_t;
    const float *lse;
    Gains gains;
    Answers answers;                   // of the rows (kAnswer)
    int32_t first;                     // vocabulary row that the piece begins with
    uint16_t *d;                       // the planes, rows of ld elements
    int64_t plane;
    int32_t ld;
};
// d's planes: float16 hi and lo, or three of bfloat16.
template <int PLANES>
__device__ __forceinline__ void planes_of(float d, uint16_t (&p)[3]) {
    if (PLANES == 3) return split3(d, p);
    _Float16 h, l;
    split(d, h, l);
    p[0] = bits(h);
    p[1] = bits(l);
}
// How the answer comes off: kTarget, one token a row, by comparison; kSpread, several tokens, from a tile of them in LDS; kLater,
// several tokens and no room for the tile, by k_subtract.
enum Answer { kTarget, kSpread, kLater };
template <class S, int PLANES, Answer ANSWER>
__global__ __launch_bounds__(S::kThreads, 2) void k_grad(const Problem p, const GradArgs e) {
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    int tm, tn, part;
    tile_of(p, blockIdx.x, tm, tn, part);
    typename S::Sums acc;
    product<S>(p, tm, tn, part, (lds_char *)lds, acc);
    const Place<S> at(tm, tn);
    const int shift_w = e.shift_w ? *e.shift_w : 0;
    __syncthreads();                               // the last stage has been read
    float *row_lse = reinterpret_cast<float *>(lds), *row_gain = row_lse + S::TM, *row_unit = row_gain + S::TM;
    int *row_target = reinterpret_cast<int *>(row_unit + S::TM);
    for (int i = threadIdx.x; i < S::TM; i += S::kThreads) {
        const int n = tm * S::TM + i;
        row_lse[i] = n < p.m ? e.lse[n] * kLog2e : 0.0f;
        const float gain = n < p.m ? e.gains.of(n) : 0.0f;
        row_gain[i] = e.many ? gain_in_d(gain) : gain;
        row_unit[i] = ldexpf(e.inv_t * kLog2e, -shift_w - (n < p.m && e.shift_x ? e.shift_x[n] : 0));
        if (ANSWER == kTarget) row_target[i] = n < p.m && e.answers.idx[n] >= e.first ? e.answers.idx[n] - e.first : -1;
    }
    float *spread = reinterpret_cast<float *>(row_target + S::TM);        // [TM][TN]: q
    if constexpr (ANSWER == kSpread) {
        static_assert((4 * S::TM + S::TM * S::TN) * 4 <= S::kLds, "room for the tile");
        for (int i = threadIdx.x; i < S::TM * S::TN; i += S::kThreads) spread[i] = 0.0f;
        __syncthreads();
        const int64_t begin = static_cast<int64_t>(tm) * S::TM * e.answers.top;
        const int entries = min(S::TM, p.m - tm * S::TM) * e.answers.top, v0 = e.first + tn * S::TN;
        for (int i = threadIdx.x; i < entries; i += S::kThreads) {
            const int32_t v = e.answers.idx[begin + i];
            if (v >= v0 && v < v0 + S::TN) spread[i / e.answers.top * S::TN + v - v0] = e.answers.q[begin + i];      // a row's entries differ
        }
    }
    __syncthreads();
    const Window d0(e.d, tm * S::TM, p.m, e.ld, 2), d1(e.d + e.plane, tm * S::TM, p.m, e.ld, 2), d2(e.d + (PLANES - 1) * e.plane, tm * S::TM, p.m, e.ld, 2);
    constexpr int kCols = S::PAIRED ? 2 : 1;       // of a store
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = at.row(i, r) - tm * S::TM;
            const float lse = row_lse[row], gain = row_gain[row], unit = row_unit[row];
            const int target = ANSWER == kTarget ? row_target[row] : -1;
#pragma unroll
            for (int j = 0; j < S::NI; j += kCols) {
                const int v = at.col(j);
                uint32_t o[3] = {0, 0, 0};
#pragma unroll
                for (int q = 0; q < kCols; ++q) {
                    const float prob = __builtin_amdgcn_exp2f(fmaf(acc[i][j + q][r], unit, -lse));
                    const float off = ANSWER == kSpread ? spread[row * S::TN + v + q - tn * S::TN] : v + q == target ? 1.0f : 0.0f;
                    const float d = gain != 0.0f && v + q < p.n ? (prob - off) * gain : 0.0f;
                    uint16_t b[3];
                    planes_of<PLANES>(d, b);
#pragma unroll
                    for (int u = 0; u < PLANES; ++u) o[u] |= static_cast<uint32_t>(b[u]) << (16 * q);
                }
                const uint32_t to = (static_cast<uint32_t>(row) * static_cast<uint32_t>(e.ld) + static_cast<uint32_t>(v)) * 2u;
                if (S::PAIRED) {
                    d0.put(to, o[0]);
                    d1.put(to, o[1]);
                    if (PLANES == 3) d2.put(to, o[2]);
                } else {
                    d0.put(to, static_cast<uint16_t>(o[0]));
                    d1.put(to, static_cast<uint16_t>(o[1]));
                    if (PLANES == 3) d2.put(to, static_cast<uint16_t>(o[2]));
                }
            }
        }
}

// The answer's part of d for the piece of the vocabulary from `first` on: entries of a row name different tokens.
template <int PLANES>
__global__ __launch_bounds__(256) void k_subtract(const Answers a, const float *gain, int many, int64_t rows, int32_t first, int32_t count, uint16_t *d, int64_t plane, int32_t ld) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= rows * a.top) return;
    const int64_t n = i / a.top;
    const int32_t at = a.idx[i] - first;
    if (a.idx[i] < 0 || at < 0 || at >= count || gain[n] == 0.0f) return;
    uint16_t *to = d + n * ld + at;
    uint16_t p[3];
    float prob = 0.0f;
#pragma unroll
    for (int u = PLANES - 1; u >= 0; --u)
        prob += PLANES == 3 ? to_float(__builtin_bit_cast(bf16, to[u * plane])) : static_cast<float>(__builtin_bit_cast(_Float16, to[u * plane]));
    planes_of<PLANES>(prob - a.q[i] * (many ? gain_in_d(gain[n]) : gain[n]), p);
#pragma unroll
    for (int u = 0; u < PLANES; ++u) to[u * plane] = p[u];
}

// dx: C[n][h] over the piece's vocabulary, added up over pieces in float32.  Where the tiles leave CUs without work the vocabulary is
// cut into shares, whose sums k_input_grad_sum adds up in a fixed order (no atomics: the same inputs give the same bits).
struct InputGradArgs {
    const int32_t *shift_w;            // many rows: d has the gain's fraction alone, W comes as scaled planes; NULL: neither
    Gains gains;
    int first, last;                   // piece
    float *sum;                        // [split][n][hidden]
    void *dx;
    int64_t lddx;
};
template <class S, typename T>
__global__ __launch_bounds__(S::kThreads, 2) void k_input_grad(const Problem p, const InputGradArgs e) {
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    int tm, tn, part;
    tile_of(p, blockIdx.x, tm, tn, part);
    typename S::Sums acc;
    product<S>(p, tm, tn, part, (lds_char *)lds, acc);
    const Place<S> at(tm, tn);
    const bool whole = p.splits == 1;
    __syncthreads();                               // the last stage has been read
    float *row_on = reinterpret_cast<float *>(lds);
    int *row_shift = reinterpret_cast<int *>(row_on + S::TM);
    const int shift_w = e.shift_w ? *e.shift_w : 0;
    for (int i = threadIdx.x; i < S::TM; i += S::kThreads) {
        const float gain = tm * S::TM + i < p.m ? e.gains.of(tm * S::TM + i) : 0.0f;
        row_on[i] = gain != 0.0f ? 1.0f : 0.0f;
        row_shift[i] = e.shift_w ? exponent_of(gain) - kTop - shift_w : 0;
    }
    __syncthreads();
    // the shares lie behind the sum over pieces
    const Window sum(e.sum + (whole ? 0 : (1 + static_cast<int64_t>(part)) * p.m * p.n), tm * S::TM, p.m, p.n, 4);
    const Window dx(e.dx, tm * S::TM, p.m, e.lddx, sizeof(T));
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int h = at.col(j);
        const bool in = h < p.n;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = at.row(i, r) - tm * S::TM, to = in ? (row * p.n + h) * 4u : kOutside;
                float v = ldexpf(acc[i][j][r], row_shift[row]);
                if (whole && !e.first) v += sum.get(to);
                if (whole && e.last) dx.put(in ? (row * static_cast<uint32_t>(e.lddx) + h) * static_cast<uint32_t>(sizeof(T)) : kOutside, static_cast<T>(row_on[row] != 0.0f ? v : 0.0f));
                else sum.put(to, v);
            }
    }
}
// The shares' sum: MANY: 64 elements a workgroup, its four waves every fourth share; else an element a thread.
template <typename T, bool MANY>
__global__ __launch_bounds__(256) void k_input_grad_sum(const InputGradArgs e, int32_t rows, int32_t hidden, int32_t splits) {
    __shared__ float part[4][64];
    constexpr int kElems = MANY ? 64 : 256, kWaves = MANY ? 4 : 1;
    const int at = threadIdx.x % kElems, wave = threadIdx.x / kElems;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kElems + at, all = static_cast<int64_t>(rows) * hidden;
    float v = 0.0f;
    if (i < all) {
#pragma unroll 4
        for (int s = wave; s < splits; s += kWaves) v += e.sum[(1 + s) * all + i];
    }
    if (MANY) {
        part[wave][at] = v;
        __syncthreads();
        v = (part[0][at] + part[1][at]) + (part[2][at] + part[3][at]);
    }
    if (wave || i >= all) return;
    if (!e.first) v += e.sum[i];
    const int64_t n = i / hidden, h = i % hidden;
    if (!e.last) e.sum[i] = v;
    else static_cast<T *>(e.dx)[n * e.lddx + h] = static_cast<T>(e.gains.of(n) != 0.0f ? v : 0.0f);
}

// dW: C[v][h] over the rows, into the caller's float32 rows.
struct WeightGradArgs {
    const int32_t *shift_x;            // many rows: x's scale, d's being kTop; NULL: neither has one
    float *dw;                         // of the piece's first row
    int accumulate;
};
template <class S>
__global__ __launch_bounds__(S::kThreads, 2) void k_weight_grad(const Problem p, const WeightGradArgs e) {
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    int tm, tn, part;
    tile_of(p, blockIdx.x, tm, tn, part);
    typename S::Sums acc;
    product<S>(p, tm, tn, part, (lds_char *)lds, acc);
    const Place<S> at(tm, tn);
    const int shift = e.shift_x ? -kTop - *e.shift_x : 0;
    const Window dw(e.dw, tm * S::TM, p.m, p.n, 4);
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int h = at.col(j);
        const bool in = h < p.n;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t to = in ? (static_cast<uint32_t>(at.row(i, r) - tm * S::TM) * p.n + h) * 4u : kOutside;
                const float d = ldexpf(acc[i][j][r], shift);
                dw.put(to, e.accumulate ? dw.get(to) + d : d);
            }
    }
}

// ------------------------------------------------------------------ few rows
// dW of up to 8 rows: a thread holds x of four columns for all rows and goes down the vocabulary, d from LDS.
// Both passes, 32768 x 2048, us, this / k_few_weight: bfloat16 1 row 150 / 161, 8 rows 148 / 154; float32 1 row 244 / 266, 8 rows 251 / 282;
// at 16 rows (4096 wide, bfloat16) 331 / 310.
constexpr int kThin = 8;
constexpr int kThinStretch = 64;       // vocabulary rows of a workgroup
template <typename T>
struct ThinWeight {
    const T *x;
    int64_t ldx;
    Gains gains;
    int32_t rows, hidden, vocab;
    const uint16_t *d;                 // three planes, rows of ld elements
    int64_t plane;
    int32_t ld;
    float *dw;
    int accumulate;
    int32_t across;                    // threads along a row of dW, a power of two up to 256
};
// WHOLE: rows of dW in 16-byte stores, four neighbouring columns a thread; else columns `across` apart.
template <typename T, int ROWS, bool WHOLE>
__global__ __launch_bounds__(256) void k_thin_weight(const ThinWeight<T> a) {
    __shared__ __attribute__((aligned(16))) float d[kThinStretch][ROWS];
    const int v0 = blockIdx.x * kThinStretch, n_v = min(kThinStretch, a.vocab - v0);
    for (int i = threadIdx.x; i < kThinStretch * ROWS; i += 256) {
        const int n = i / kThinStretch, v = i % kThinStretch;              // neighbours along a row of d
        const uint16_t *from = a.d + static_cast<int64_t>(n) * a.ld + v0 + v;
        float s = 0.0f;
        if (n < a.rows && v < n_v)
#pragma unroll
            for (int q = 2; q >= 0; --q) s += to_float(__builtin_bit_cast(bf16, from[q * a.plane]));
        d[v][n] = s;
    }
    const int tx = threadIdx.x & (a.across - 1), ty = threadIdx.x / a.across, down = 256 / a.across;
    const int c0 = blockIdx.y * a.across * 4 + (WHOLE ? 4 * tx : tx), step = WHOLE ? 1 : a.across;
    float x[ROWS][4];
#pragma unroll
    for (int n = 0; n < ROWS; ++n) {
        const bool in = n < a.rows && a.gains.of(n) != 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = in && c0 + e * step < a.hidden ? to_float(a.x[n * a.ldx + c0 + e * step]) : 0.0f;
    }
    __syncthreads();
    for (int v = ty; v < n_v; v += down) {
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < ROWS; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fmaf(d[v][n], x[n][e], s[e]);
        float *to = a.dw + static_cast<int64_t>(v0 + v) * a.hidden + c0;
        if (WHOLE) {
            if (c0 < a.hidden) {
                float4 o = make_float4(s[0], s[1], s[2], s[3]);
                if (a.accumulate) {
                    const float4 was = *reinterpret_cast<const float4 *>(to);
                    o = make_float4(was.x + o.x, was.y + o.y, was.z + o.z, was.w + o.w);
                }
                *reinterpret_cast<float4 *>(to) = o;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c0 + e * step < a.hidden) to[e * step] = a.accumulate ? to[e * step] + s[e] : s[e];
        }
    }
}

// ------------------------------------- few rows, W not as the loads to LDS want it
// Measured, us (bytes of W, or of dW, a second): 65536 x 4224 float32 under 107 tokens, logits 404 (2.7 TB/s; six products of 59 GFLOP:
// 0.87 PFLOP/s); 28774 x 3220 float32 under 48, logits 145 (2.6), d 129 (2.9), dx 114 (3.3), dW 141 (2.6); 16384 x 5907 float32 under 18,
// logits 135 (2.9), d 111 (3.5), dx 78 (5.0), dW 114 (3.4); 65536 x 4451 bfloat16, odd, under 74, logits 227 (2.6), d 189 (3.1), dx 407
// (1.4), dW 482 (2.4).  Bound by memory, and by how little of a row a load takes (32 rows of 32 to 64 bytes each): bfloat16 rows that
// go to LDS instead, 128 bytes at a time, are read at 4 to 5 TB/s (32768 x 4096 under 16 tokens 47 us, through registers 96), so that
// way is kept for those that can.
// Float32, and bfloat16 rows of any alignment: W comes straight from memory to registers, is split into planes there, and is
// neither copied nor gone over beforehand.  A share of the matrix instructions' operands is thus read by one wave alone; x (or d),
// small, is laid out before and shared.
template <typename T> constexpr int kPlanesOf = sizeof(T) == 4 ? 3 : 1;
// Eight elements in three planes whose sum they are: 8 bits cut off, which cannot leave the range, the next 8 rounded, so that what
// the products leave out has no sign of its own, the rest.  Infinities come out as NaN.
__device__ __forceinline__ void cut3(const float (&v)[8], bfloat8 (&p)[3]) {
    uint32_t o[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t h[2], l[2];
        float rest[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float x = v[2 * e + u];
            h[u] = __builtin_bit_cast(uint32_t, x);
            rest[u] = x - __builtin_bit_cast(float, h[u] & 0xffff0000u);
        }
        const uint32_t m = static_cast<uint32_t>(bits(static_cast<bf16>(rest[0]))) | static_cast<uint32_t>(bits(static_cast<bf16>(rest[1]))) << 16;
        l[0] = __builtin_bit_cast(uint32_t, rest[0] - __builtin_bit_cast(float, m << 16));
        l[1] = __builtin_bit_cast(uint32_t, rest[1] - __builtin_bit_cast(float, m & 0xffff0000u));
        o[0][e] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302u);                    // the upper halves
        o[1][e] = m;
        o[2][e] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302u);
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) __builtin_memcpy(&p[q], o[q], 16);
}
// bfloat16 rows of any alignment: 16-byte loads that are not aligned to 4 bytes take about twice as long, so the words that hold the
// elements are loaded, and one more where they begin in a word's upper half; `joints` puts them together when they are needed.
__device__ __forceinline__ uint32_t joint(const void *at) { return reinterpret_cast<uintptr_t>(at) & 2 ? 0x05040302u : 0x03020100u; }
__device__ __forceinline__ const uint32_t *word_of(const bf16 *at) { return reinterpret_cast<const uint32_t *>(reinterpret_cast<uintptr_t>(at) & ~static_cast<uintptr_t>(3)); }
// FRAGS times eight consecutive elements of a row: those of the wave's lower and upper half in turn.
template <typename T, int FRAGS> struct Stretch;
template <int FRAGS> struct Stretch<float, FRAGS> {
    static constexpr int kLoads = 2 * FRAGS;
    float v[FRAGS][8];
    __device__ __forceinline__ void load(const float *at) {
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) __builtin_memcpy(v[f], at + 16 * f, 32);
    }
    __device__ __forceinline__ void planes(bfloat8 (&p)[FRAGS][3], uint32_t) const {
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) cut3(v[f], p[f]);
    }
};
template <int FRAGS> struct Stretch<bf16, FRAGS> {
    static constexpr int kLoads = FRAGS + 1;
    uint32_t w[FRAGS][4], more;        // more: the word behind the last eight
    __device__ __forceinline__ void load(const bf16 *at) {
        const uint32_t *words = word_of(at);
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) __builtin_memcpy(w[f], words + 8 * f, 16);
        more = words[8 * (FRAGS - 1) + (reinterpret_cast<uintptr_t>(at) & 2 ? 4 : 3)];      // no word without an element of these
    }
    __device__ __forceinline__ void planes(bfloat8 (&p)[FRAGS][1], uint32_t joints) const {
        const bool upper = threadIdx.x & 32;
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            // the word behind a lower half's eight is the upper half's first, behind that one's the lower half's next
            uint32_t behind = more;
            if (f + 1 < FRAGS) {
                const auto both = __builtin_amdgcn_permlane32_swap(w[f][0], w[f + 1][0], false, false);
                behind = upper ? both[0] : both[1];
            } else {
                const auto both = __builtin_amdgcn_permlane32_swap(w[f][0], w[f][0], false, false);
                behind = upper ? more : both[1];
            }
            const uint32_t o[4] = {__builtin_amdgcn_perm(w[f][1], w[f][0], joints), __builtin_amdgcn_perm(w[f][2], w[f][1], joints),
                                   __builtin_amdgcn_perm(w[f][3], w[f][2], joints), __builtin_amdgcn_perm(behind, w[f][3], joints)};
            __builtin_memcpy(&p[f][0], o, 16);
        }
    }
};
// Eight elements as planes.
__device__ __forceinline__ void planes_of_eight(const float (&v)[8], bfloat8 (&p)[3]) { cut3(v, p); }
__device__ __forceinline__ void planes_of_eight(const bf16 (&v)[8], bfloat8 (&p)[1]) { __builtin_memcpy(&p[0], v, 16); }

template <typename T>
struct FewLogits {
    const T *w;
    int64_t ldw;
    float inv_t;
    // forward
    float2 *stats;                     // [n][strips of 32 vocabulary rows]
    int32_t strips, first_strip;
    Picked picked;
    // backward
    const float *lse;
    Gains gains;
    Answers answers;
    int32_t first;                     // vocabulary row that the piece begins with
    uint16_t *d;                       // three planes, rows of ld elements
    int64_t plane;
    int32_t ld;
};
// What becomes of the logits: a maximum and a sum, and an answer's own logits, of one token (kStats) or several (kTaught), or d of an
// answer of one (kOne) or several tokens (kMore).
enum Purpose { kStats, kTaught, kOne, kMore };
// k of a stage that a wave takes
template <typename T, int NB, int WK> constexpr int kFewStage = (sizeof(T) == 4 && (NB > 1 || WK > 1) ? 32 : 64) / (WK == 1 ? 1 : 2);
// p: C[v][n], b: x's planes.  A wave takes 32 vocabulary rows and NB * 32 tokens; WK of a workgroup's four waves share the k axis of
// these, the others stand side by side; x in a ring of three stages.
template <typename T, int NB, int WK, Purpose FOR>
__global__ __launch_bounds__(256, WK == 4 && NB == 4 ? 1 : 2) void k_few_logits(const Problem p, const FewLogits<T> e) {
    constexpr int P = kPlanesOf<T>, kMine = kFewStage<T, NB, WK>, KS = kMine * WK, kN = NB * 32, kM = 128 / WK, kPlane = kN * KS * 2, kStage = P * kPlane, kFrags = kMine / 16;
    constexpr int kSpread = FOR == kMore || FOR == kTaught ? kM * kN * 4 : 0, kLds = kSpread > 3 * kStage ? kSpread : 3 * kStage;
    static_assert(WK == 1 || 2 * kN * 32 * 4 <= kLds, "room for two waves' sums");
    using Load = Loader<false, kN, 256, false, KS>;
    __shared__ __attribute__((aligned(16))) char lds_room[kLds];
    lds_char *lds = (lds_char *)lds_room;
    int tm, tn, part;
    tile_of(p, blockIdx.x, tm, tn, part);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int v0 = tm * kM + wave / WK * 32, mine = wave % WK * kMine;
    const T *row = e.w + static_cast<int64_t>(min(v0 + (lane & 31), p.m - 1)) * e.ldw + mine + 8 * half;     // rows beyond the last repeat it
    const uint32_t joints = joint(row);
    Load load;
    load.init(tid, p.b.ld);
    Reader<false, kN, NB, false, KS> read;
    read.init(0, lane, mine / 16);
    Source<false, KS> x;
    x.init(p.b, tn * kN, p.n, 0, p.k);
    auto next_x = [&](int to) {
#pragma unroll
        for (int q = 0; q < P; ++q) load.issue(x.at + q * p.b.plane, x.bytes(), x.k_left, lds + to + q * kPlane, wave);
        x.advance();
    };
    const int whole = p.k / KS;
    auto next_w = [&](Stretch<T, kFrags> &to, int s) { to.load(row + min(s, whole - 1) * KS); };        // behind the last whole stage that one again
    float16v acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
    constexpr bool kSmall = P > 1 && NB < 4;                         // the small products have sums of their own: one rounding of the large one in 16 k
    float16v small[kSmall ? NB : 1];
    if (kSmall)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) small[kSmall ? j : 0][r] = 0.0f;
    auto multiply = [&](const bfloat8 (&a)[kFrags][P], int slot) {
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            bfloat8 b[P][NB];
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int j = 0; j < NB; ++j) b[q][j] = read.template read<bfloat8>(lds + slot + q * kPlane, j, f);
#pragma unroll
            for (int t = 0; t < Terms<P, P>::n; ++t)
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    float16v &to = kSmall && t + 1 < Terms<P, P>::n ? small[kSmall ? j : 0] : acc[j];
                    to = mfma(a[f][Terms<P, P>::a[t]], b[Terms<P, P>::b[t]][j], to);
                }
        }
    };
    constexpr int kLoadsX = P * Load::kLoads, kLoadsW = Stretch<T, kFrags>::kLoads;
    Stretch<T, kFrags> w[2];
    next_x(0);
    if (whole) next_w(w[0], 0);
    __builtin_amdgcn_sched_barrier(0);
    next_x(kStage);
    if (whole) next_w(w[1], 1);
    __builtin_amdgcn_sched_barrier(0);
    int now = 0, then = 2 * kStage;
    // Stage s: x and W of s are here when only those of s + 1 are on their way; behind the barrier all waves have x of s, and have
    // read x of s - 1, whose place x of s + 2 takes.
    auto stage = [&](int s, Stretch<T, kFrags> &mine) {
        __builtin_amdgcn_s_waitcnt(wait_for(kLoadsX + kLoadsW, 15));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        bfloat8 a[kFrags][P];
        mine.planes(a, joints);
        next_x(then);
        next_w(mine, s + 2);
        __builtin_amdgcn_sched_barrier(0);
        multiply(a, now);
        __builtin_amdgcn_s_waitcnt(wait_for(63, 0));         // read
        __builtin_amdgcn_sched_barrier(0);
        then = now;
        now = now == 2 * kStage ? 0 : now + kStage;
    };
    int s = 0;
    for (; s + 2 <= whole; s += 2) {
        stage(s, w[0]);
        stage(s + 1, w[1]);
    }
    if (s < whole) stage(s, w[0]);
    __builtin_amdgcn_s_waitcnt(wait_for(0, 0));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (whole * KS < p.k) {                                          // the rows' ends
        bfloat8 a[kFrags][P];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int k = whole * KS + 16 * f;
            T q[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) q[u] = k + mine + 8 * half + u < p.k ? row[k + u] : static_cast<T>(0.0f);
            planes_of_eight(q, a[f]);
        }
        multiply(a, now);
    }
    if constexpr (kSmall)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[j] += small[j];
    if constexpr (WK > 1) {                                          // the waves' sums, folded in halves
        static_assert(WK == 4, "one tile a workgroup");
        float *tile = reinterpret_cast<float *>(lds_room);           // [2][NB * 16][lane]
        for (int to = 2; to; to /= 2) {
            __syncthreads();
            if (wave >= to && wave < 2 * to)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) tile[(((wave - to) * NB + j) * 16 + r) * 64 + lane] = acc[j][r];
            __syncthreads();
            if (wave < to)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[j][r] += tile[((wave * NB + j) * 16 + r) * 64 + lane];
        }
    }
    const bool last = WK == 1 || wave == 0;                          // holds the sums
    if constexpr (FOR == kStats || FOR == kTaught) {
        const bool here = v0 < p.m && last;
        if (FOR == kStats && !here) return;
        float *tile = reinterpret_cast<float *>(lds_room);           // kTaught: [kM][kN], the logits
        if (FOR == kTaught) __syncthreads();                         // the last stage has been read
        if (here)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int n = tn * kN + 32 * j + (lane & 31);
            float most = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                acc[j][r] = v0 + 8 * (r >> 2) + 4 * half + (r & 3) < p.m ? acc[j][r] * e.inv_t : -INFINITY;
                most = fmaxf(most, acc[j][r]);
            }
            if (FOR == kTaught) {
#pragma unroll
                for (int r = 0; r < 16; ++r) tile[(v0 - tm * kM + 8 * (r >> 2) + 4 * half + (r & 3)) * kN + 32 * j + (lane & 31)] = acc[j][r];
            } else {
                const int32_t target = n < p.n ? e.picked.target[n] : -1, from = e.picked.first + v0;
                if (target >= from && target < e.picked.first + min(p.m, v0 + 32)) {                // rare
                    const int own = target - from - 4 * half;        // one of the wave's halves has it
                    float logit = 0.0f;
                    most = -INFINITY;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool it = 8 * (r >> 2) + (r & 3) == own;
                        logit = it ? acc[j][r] : logit;
                        acc[j][r] = it ? -INFINITY : acc[j][r];
                        most = fmaxf(most, acc[j][r]);
                    }
                    if (((target - from) >> 2 & 1) == half) e.picked.logit[n] = logit;
                }
            }
            most = fmaxf(most, __shfl_xor(most, 32));
            const float around = most > -INFINITY ? most : 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[j][r] - around) * kLog2e);
            sum += __shfl_xor(sum, 32);
            if (half == 0 && n < p.n) e.stats[static_cast<int64_t>(n) * e.strips + e.first_strip + v0 / 32] = make_float2(most, sum);
        }
        if constexpr (FOR == kTaught) {
            __syncthreads();
            pick<256>(e.picked, tn * kN, min(kN, p.n - tn * kN), e.picked.first + tm * kM, max(0, min(kM, p.m - tm * kM)), [&](int n, int v) { return tile[v * kN + n]; });
        }
    } else {
        float *spread = reinterpret_cast<float *>(lds_room);         // [kM][kN]: q
        if constexpr (FOR == kMore) {
            __syncthreads();                                         // the last stage has been read
            for (int i = tid; i < kM * kN; i += 256) spread[i] = 0.0f;
            __syncthreads();
            const int64_t begin = static_cast<int64_t>(tn) * kN * e.answers.top;
            const int entries = min(kN, p.n - tn * kN) * e.answers.top, from = e.first + tm * kM;
            for (int i = tid; i < entries; i += 256) {
                const int32_t v = e.answers.idx[begin + i];
                if (v >= from && v < from + kM) spread[(v - from) * kN + i / e.answers.top] = e.answers.q[begin + i];      // a row's entries differ
            }
            __syncthreads();
        }
        if (!last) return;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int n = tn * kN + 32 * j + (lane & 31);
            if (n >= p.n) continue;
            const float gain = e.gains.of(n), lse = e.lse[n] * kLog2e;
            const int32_t target = FOR == kOne && e.answers.idx[n] >= e.first ? e.answers.idx[n] - e.first : -1;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint16_t o[3][4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int v = v0 + 8 * g + 4 * half + u;
                    const float prob = __builtin_amdgcn_exp2f(fmaf(acc[j][4 * g + u], e.inv_t * kLog2e, -lse));
                    const float off = FOR == kMore ? spread[(v - tm * kM) * kN + 32 * j + (lane & 31)] : v == target ? 1.0f : 0.0f;
                    uint16_t b[3];
                    split3(gain != 0.0f && v < p.m ? (prob - off) * gain : 0.0f, b);
#pragma unroll
                    for (int q = 0; q < 3; ++q) o[q][u] = b[q];
                }
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    *reinterpret_cast<uint2 *>(e.d + q * e.plane + static_cast<int64_t>(n) * e.ld + v0 + 8 * g + 4 * half) = *reinterpret_cast<const uint2 *>(o[q]);
            }
        }
    }
}

// dx in shares of the vocabulary, 64 tokens by 128 columns a workgroup.  A lane loads four neighbouring columns of eight vocabulary
// rows, k of its half of a fragment, for the same place in four blocks of 32 columns; the waves take every fourth 16 rows.
template <typename T>
struct FewInput {
    const T *w;
    int64_t ldw;
    const uint16_t *d;                 // planes, rows of ld elements
    int64_t plane;
    int32_t ld;
    int32_t rows, hidden, vocab, share;    // share: vocabulary rows of a workgroup, a multiple of 64
    float *sum;                            // [1 + share's number][n][hidden]
    Problem p;                             // m: blocks of columns by shares, n: groups of tokens
    int32_t across;                        // blocks of columns
};
// Four columns of eight rows as they are loaded, and a column of these as a fragment.  joints: of the even and the odd rows.
template <typename T> struct Four;
template <> struct Four<float> {
    float v[8][4];
    // rows: the first of the eight and on, uniform; lane: a lane's elements behind
    struct Lane {
        uint32_t at;
        __device__ __forceinline__ Lane(const float *, int64_t, uint32_t lane) : at(lane) {}
    };
    __device__ __forceinline__ void load(int u, const float *row, const Lane &lane) { __builtin_memcpy(v[u], row + lane.at, 16); }
    __device__ __forceinline__ void set(int u, const float (&q)[4]) { __builtin_memcpy(v[u], q, 16); }
    __device__ __forceinline__ void clear(int u) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] = 0.0f;
    }
    __device__ __forceinline__ void column(int e, bfloat8 (&p)[3], const uint32_t (&)[2]) const {
        const float q[8] = {v[0][e], v[1][e], v[2][e], v[3][e], v[4][e], v[5][e], v[6][e], v[7][e]};
        cut3(q, p);
    }
};
template <> struct Four<bf16> {
    uint32_t w[8][3];
    // in a row of even and of odd number: the byte offset of a lane's first word and of its last from the row's first word
    struct Lane {
        uint32_t word[2], last[2];
        __device__ __forceinline__ Lane(const bf16 *first, int64_t ld, uint32_t lane) {
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(first + odd * ld) & 2) + 2 * lane;
                word[odd] = at & ~3u;
                last[odd] = word[odd] + (at & 2 ? 8 : 4);            // no word without an element of these
            }
        }
    };
    __device__ __forceinline__ void load(int u, const bf16 *row, const Lane &lane) {
        const char *words = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(row) & ~static_cast<uintptr_t>(3));
        __builtin_memcpy(w[u], words + lane.word[u & 1], 8);
        __builtin_memcpy(&w[u][2], words + lane.last[u & 1], 4);
    }
    __device__ __forceinline__ void set(int u, const bf16 (&q)[4]) { __builtin_memcpy(w[u], q, 8); }
    __device__ __forceinline__ void clear(int u) { w[u][0] = w[u][1] = w[u][2] = 0; }
    __device__ __forceinline__ void column(int e, bfloat8 (&p)[1], const uint32_t (&joints)[2]) const {
        uint32_t o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t even = __builtin_amdgcn_perm(w[2 * u][e / 2 + 1], w[2 * u][e / 2], joints[0]);
            const uint32_t odd = __builtin_amdgcn_perm(w[2 * u + 1][e / 2 + 1], w[2 * u + 1][e / 2], joints[1]);
            o[u] = __builtin_amdgcn_perm(odd, even, e % 2 ? 0x07060302u : 0x05040100u);
        }
        __builtin_memcpy(&p[0], o, 16);
    }
};
// NARROW: fewer than four columns in all, loaded one by one.
template <typename T, int NB, bool NARROW>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void k_few_input(const FewInput<T> a) {
    constexpr int P = kPlanesOf<T>, D = P == 3 ? 3 : 2;              // bfloat16, the result's type: two planes of d are good to 2^-18, a float32 sum's error
    __shared__ float tile[2][32 * NB][128 + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    int at, group, part;
    tile_of(a.p, blockIdx.x, at, group, part);                       // the groups of tokens that read the same of W beside one another
    const int n0 = group * 32 * NB, c0 = at % a.across * 128, number = at / a.across;
    const int c = NARROW ? 0 : min(c0 + 4 * (lane & 31), a.hidden - 4);      // columns beyond the last: those before once more
    const int begin = number * a.share, end = min(a.vocab, begin + a.share), whole = begin + (end - begin) / 16 * 16;
    // a lane's rows are 8 * half + u of 16 from `begin`, a multiple of 64, on: whether u is even tells where in a word they begin
    const uint32_t joints[2] = {NARROW ? joint(nullptr) : joint(a.w + c), NARROW ? joint(nullptr) : joint(a.w + a.ldw + c)};
    float16v acc[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][b][r] = 0.0f;
    struct Turn {
        Four<T> w;
        bfloat8 d[D][NB];
    };
    const uint32_t lane_at = static_cast<uint32_t>(8 * half) * static_cast<uint32_t>(a.ldw) + c;
    const typename Four<T>::Lane in_rows(a.w, a.ldw, lane_at);
    const uint16_t *d_at[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) d_at[i] = a.d + static_cast<int64_t>(min(n0 + 32 * i + (lane & 31), a.rows - 1)) * a.ld + 8 * half;
    auto fetch = [&](Turn &t, int v, bool end) {                     // 16 rows from v on; at the end, those beyond the last repeat it
        const T *first = a.w + static_cast<int64_t>(v) * a.ldw;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (NARROW || end) {
                const T *from = a.w + static_cast<int64_t>(min(v + 8 * half + u, a.vocab - 1)) * a.ldw + c;
                T q[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = from[min(e, a.hidden - 1)];
                t.w.set(u, q);
            } else {
                t.w.load(u, first + u * a.ldw, in_rows);
            }
        }
#pragma unroll
        for (int q = 0; q < D; ++q)
#pragma unroll
            for (int i = 0; i < NB; ++i) t.d[q][i] = *reinterpret_cast<const bfloat8 *>(d_at[i] + q * a.plane + v);
    };
    auto multiply = [&](const Turn &t, const uint32_t (&joints)[2]) {
        using P2 = Terms<D, P>;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            bfloat8 w[P];
            t.w.column(b, w, joints);
#pragma unroll
            for (int k = 0; k < P2::n; ++k)
#pragma unroll
                for (int i = 0; i < NB; ++i) acc[i][b] = mfma(t.d[P2::a[k]][i], w[P2::b[k]], acc[i][b]);
        }
    };
    // whole turns; behind the last one that one is loaded again
    int v = begin + 16 * wave;
    const int most = whole - 16;
    Turn t[2];
    if (v < whole) {
        fetch(t[0], v, false);
        for (; v + 64 < whole; v += 128) {                           // two at a time
            fetch(t[1], v + 64, false);
            multiply(t[0], joints);
            fetch(t[0], min(v + 128, most), false);
            multiply(t[1], joints);
        }
        if (v < whole) {
            multiply(t[0], joints);
            v += 64;
        }
    }
    if (v < end) {                                                   // the last rows, fewer than 16: the others count nothing, whatever they hold
        fetch(t[0], v, true);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (v + 8 * half + u >= end) t[0].w.clear(u);
        const uint32_t straight[2] = {joint(nullptr), joint(nullptr)};
        multiply(t[0], straight);
    }
    // C[n][column]: the four waves' sums, folded in halves; the first wave's come last
    for (int to = 2; to >= 0; to /= 2) {
        if (wave >= to && wave < (to ? 2 * to : 1))
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) tile[wave - to][32 * i + 8 * (r >> 2) + 4 * half + (r & 3)][4 * (lane & 31) + b] = acc[i][b][r];
        __syncthreads();
        if (to == 0) break;
        if (wave < to)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][b][r] += tile[wave][32 * i + 8 * (r >> 2) + 4 * half + (r & 3)][4 * (lane & 31) + b];
        __syncthreads();
    }
    float *out = a.sum + ((1 + static_cast<int64_t>(number)) * a.rows + n0) * a.hidden;
    for (int i = threadIdx.x; i < min(32 * NB, a.rows - n0) * 128; i += 256) {
        const int n = i / 128, col = c0 + i % 128;
        // a lane whose columns would leave the row holds the row's last four
        const int lane_of = (i % 128) / 4, held = NARROW ? 0 : min(c0 + 4 * lane_of, a.hidden - 4);
        if (col < a.hidden) out[static_cast<int64_t>(n) * a.hidden + col] = tile[0][n][4 * lane_of + (col - held)];
    }
}

// dW of 9 to 128 rows: all that it does beside writing is little, so a wave keeps x of its columns in registers, as fragments for
// all rows, and goes down the vocabulary; d comes through LDS in blocks of 64 vocabulary rows.  CB: neighbouring columns a lane
// holds, one in each of as many blocks of 32, so that a store takes 4 * CB bytes.
template <typename T>
struct FewWeight {
    const T *x;
    int64_t ldx;
    Gains gains;
    float *dw;
    int accumulate;
    int32_t stretch;                   // vocabulary rows of a workgroup, a multiple of 64
};
// p: a: d's planes, [n][v]; m vocabulary rows, n columns, k rows of x (up to 16 * STEPS).
template <typename T, int STEPS, int CB>
__global__ __launch_bounds__(256, 2) void k_few_weight(const Problem p, const FewWeight<T> e) {
    constexpr int P = kPlanesOf<T>, kRows = 16 * STEPS, kPlane = 64 * kRows * 2, kBlock = 3 * kPlane, kBuf = STEPS <= 4 ? 2 : 1;
    using Load = Loader<true, 64, 256, false, kRows>;
    __shared__ __attribute__((aligned(16))) char lds_room[kBuf * kBlock];
    lds_char *lds = (lds_char *)lds_room;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int first = blockIdx.x * e.stretch, last = min(p.m, first + e.stretch);
    const int c = (blockIdx.y * 4 + wave) * 32 * CB + CB * (lane & 31);
    const bool writes = (blockIdx.y * 4 + wave) * 32 * CB < p.n;
    Load load;
    load.init(tid, p.a.ld);
    Reader<true, 64, 2, false, kRows> read;
    read.init(0, lane);
    auto next = [&](int v, int to) {
        Source<true, kRows> d;
        d.init(p.a, v, p.m, 0, p.k);
#pragma unroll
        for (int q = 0; q < 3; ++q) load.issue(d.at + q * p.a.plane, v < last ? d.bytes() : 0u, p.k, lds + to + q * kPlane, wave);
    };
    next(first, 0);
    bfloat8 x[STEPS][CB][P];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        T raw[CB][8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int n = 16 * k + 8 * half + u;
            const bool in = n < p.k && e.gains.of(n) != 0.0f;
#pragma unroll
            for (int b = 0; b < CB; ++b) raw[b][u] = in ? e.x[n * e.ldx + min(c + b, p.n - 1)] : static_cast<T>(0.0f);
        }
#pragma unroll
        for (int b = 0; b < CB; ++b) planes_of_eight(raw[b], x[k][b]);
    }
    const uint32_t lane_at = static_cast<uint32_t>(4 * half) * static_cast<uint32_t>(p.n) + c;
    int now = 0;
    for (int v0 = first; v0 < last; v0 += 64) {
        const bool full = v0 + 64 <= last;
        if (kBuf == 1 && v0 > first) {
            __builtin_amdgcn_s_barrier();                            // the block before has been read by all
            __builtin_amdgcn_sched_barrier(0);
            next(v0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the block's loads are older than the stores of the block before, 32 at least in a wave that has columns
        if (kBuf == 2 && writes && v0 > first) __builtin_amdgcn_s_waitcnt(wait_for(32, 15));
        else __builtin_amdgcn_s_waitcnt(wait_for(0, 15));
        __builtin_amdgcn_s_barrier();                                // the block is here, the one before has been read by all
        __builtin_amdgcn_sched_barrier(0);
        if (kBuf == 2) next(v0 + 64, kBlock - now);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float16v acc[CB];
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                bfloat8 d[3];
#pragma unroll
                for (int q = 0; q < 3; ++q) d[q] = read.template read<bfloat8>(lds + now + q * kPlane, i, k);
                using P2 = Terms<3, P>;
#pragma unroll
                for (int t = 0; t < P2::n; ++t)
#pragma unroll
                    for (int b = 0; b < CB; ++b) acc[b] = mfma(d[P2::a[t]], x[k][b][P2::b[t]], acc[b]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int v = v0 + 32 * i + 8 * (r >> 2) + (r & 3);      // and 4 * half
                float *to = e.dw + static_cast<int64_t>(v) * p.n + lane_at;
                const bool in = full || v + 4 * half < last;
                float o[CB];
#pragma unroll
                for (int b = 0; b < CB; ++b) o[b] = acc[b][r];
                if (in && c + CB <= p.n) {
                    if (e.accumulate) {
                        float was[CB];
                        __builtin_memcpy(was, to, sizeof(was));
#pragma unroll
                        for (int b = 0; b < CB; ++b) o[b] += was[b];
                    }
                    __builtin_memcpy(to, o, sizeof(o));
                } else if (in) {
#pragma unroll
                    for (int b = 0; b < CB; ++b)
                        if (c + b < p.n) to[b] = e.accumulate ? to[b] + o[b] : o[b];
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(wait_for(63, 0));                 // read
        __builtin_amdgcn_sched_barrier(0);
        if (kBuf == 2) now = kBlock - now;
    }
    __builtin_amdgcn_s_waitcnt(wait_for(0, 0));                      // nothing is on its way to LDS any more
}

// ---- host side ---------------------------------------------------------------
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
constexpr unsigned blocks_for(int64_t n, int64_t most) { return static_cast<unsigned>(n < most ? n : most); }
constexpr int64_t kPlaneBlocks = 4096;
constexpr int kStep = 64;              // k in whose multiples the k axis is cut

// Tiles of a product.  256 x 256: a workgroup of eight waves per CU; 128 x 128: two of four waves; 64 x 64: two of four waves
// with a deep ring, for products with little to do.  64 x 256 with a deep ring: dx of up to 64 rows, which reads W across its rows,
// 512 bytes of each instead of 128.
enum Tile { kTile64, kTile128, kTile256, kTileWide };
constexpr int64_t kSide[] = {64, 128, 256};        // of the square ones
constexpr int64_t kMaxTiles = int64_t(1) << 22;    // of a launch, up to 512 threads each
struct Choice {
    Tile tile;
    int64_t splits;
};
// Both passes, us, with the largest tile 256 / 128 / 64: bfloat16 10007 x 1000 under 777 rows 181 / 204 / 256, 50021 x 2048
// under 4096 4317 / 5504 / 9312; a unit of 2.5 instead of 3 for 64: float32 4096 x 2048 under 1024 rows 349 for 301.
// A round over all CUs takes so many units of time per stage of 64 k (measured: the larger tiles move fewer bytes per product,
// the small ones leave fewer CUs without work).  The k axis is cut into shares where the tiles alone do not fill the CUs.
Choice choose(int64_t m, int64_t n, int64_t k, int64_t splits_most, Tile largest = kTile256) {
    Choice best = {};
    double least = 0.0;
    for (int tile = kTile64; tile <= largest; ++tile) {
        static constexpr int64_t kRoom[] = {512, 512, 256};
        static constexpr double kUnits[] = {3.0, 5.0, 8.0};
        const int64_t t = kSide[tile], room = kRoom[tile], steps = (k + kStep - 1) / kStep;
        if (tile > kTile64 && std::min(m, n) <= t / 2) break;         // half of it and more would be beyond the edge
        const int64_t tiles = ((m + t - 1) / t) * ((n + t - 1) / t), splits = std::max<int64_t>(1, std::min({splits_most, room / tiles, steps}));
        const double cost = static_cast<double>((tiles * splits + room - 1) / room) * (static_cast<double>((steps + splits - 1) / splits) + 4.0) * kUnits[tile];
        if (tile == kTile64 || cost < least) { least = cost; best = {static_cast<Tile>(tile), splits}; }
    }
    return best;
}
// Stages of 64 k, or of 32 where an operand has several planes.
template <Tile TILE, typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB> struct ShapeOf;
template <typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB>
struct ShapeOf<kTile64, V, A_MC, B_MC, PAIRED, PA, PB> { using S = Shape<V, A_MC, B_MC, 64, 64, 2, 2, false, PA, PB, PA * PB >= 3 ? 32 : 64, true>; };
template <typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB>
struct ShapeOf<kTile128, V, A_MC, B_MC, PAIRED, PA, PB> { using S = Shape<V, A_MC, B_MC, 128, 128, 2, 2, PAIRED, PA, PB, PA * PB >= 2 ? 32 : 64, false>; };
template <typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB>
struct ShapeOf<kTile256, V, A_MC, B_MC, PAIRED, PA, PB> { using S = Shape<V, A_MC, B_MC, 256, 256, 2, 4, PAIRED, PA, PB, PA * PB >= 2 ? 32 : 64, false>; };
template <typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB>
struct ShapeOf<kTileWide, V, A_MC, B_MC, PAIRED, PA, PB> { using S = Shape<V, A_MC, B_MC, 64, 256, 1, 4, false, PA, PB, 32, true>; };
constexpr int kStripOf[] = {32, 64, 128};          // vocabulary rows of a strip: a wave's of k_stats

Problem problem(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k) {
    Problem p = {};
    p.a = a;
    p.b = b;
    p.m = static_cast<int32_t>(m);
    p.n = static_cast<int32_t>(n);
    p.k = static_cast<int32_t>(k);
    return p;
}
template <class S>
dim3 cut(Problem &p, int64_t splits) {
    p.m_tiles = (p.m + S::TM - 1) / S::TM;
    p.n_tiles = (p.n + S::TN - 1) / S::TN;
    p.split_k = static_cast<int32_t>(up((p.k + splits - 1) / splits, kStep));
    p.splits = (p.k + p.split_k - 1) / p.split_k;
    return dim3(static_cast<unsigned>(p.m_tiles) * p.n_tiles * p.splits);
}
// f(shape) for the tile chosen; three planes go with few rows, two of both operands with many.
template <typename V, bool A_MC, bool B_MC, bool PAIRED, int PA, int PB, typename F>
void with_shape(Tile tile, F &&f) {
    if (tile == kTile64) return f(typename ShapeOf<kTile64, V, A_MC, B_MC, PAIRED, PA, PB>::S{});
    if constexpr (!A_MC && B_MC && PA == 2 && PB == 1 && std::is_same<V, bfloat8>::value)       // few rows
        if (tile == kTileWide) return f(typename ShapeOf<kTileWide, V, A_MC, B_MC, PAIRED, PA, PB>::S{});
    if constexpr (PA < 3) {
        if (tile == kTile128) return f(typename ShapeOf<kTile128, V, A_MC, B_MC, PAIRED, PA, PB>::S{});
        f(typename ShapeOf<kTile256, V, A_MC, B_MC, PAIRED, PA, PB>::S{});
    }
}

// How a call is cut up.
struct Layout {
    bool few;                          // the form for few rows
    bool direct;                       // ... with W straight from memory to registers
    int64_t rows;                      // of a row chunk
    int64_t ld;                        // of planes of x and W
    int64_t piece;                     // vocabulary rows at a time, a multiple of 256
    int32_t splits_most;               // shares of dx's k axis that there is room for
    Tile stats_tile;
    int32_t strips;
    int32_t share;                     // direct: vocabulary rows of a share of dx
    int64_t x_plane, w_plane, d_plane; // elements from one plane to the next
    // offsets in the workspace
    size_t idx, q, stats, picked, gain, shifts, parts_x, parts_w, shift_rows, x, x_raw, w, d, sum, total;
};

// Whether dx of few rows takes the wide tile.  Both passes over 32768 rows of W, us, wide / 64 x 64: 40 tokens 4096 wide 334 / 349,
// 64 tokens 351 / 368; 40 tokens 1024 wide 103 / 99, 512 wide 80 / 71 (too few tiles).
bool wide_dx(int32_t dtype, int64_t rows, int64_t hidden) { return dtype == RSDGC_BF16 && rows <= 64 && hidden >= 2048; }

// Vocabulary rows of a share of dx, of 64 tokens by 128 columns a workgroup: 512 workgroups, as far as a share has 256 rows.
int32_t few_share(int64_t rows, int64_t hidden, int64_t vocab) {
    const int64_t across = (hidden + 127) / 128 * ((std::max<int64_t>(1, rows) + 63) / 64);
    const int64_t shares = std::max<int64_t>(1, std::min(512 / across, vocab / 256));
    return static_cast<int32_t>(up((vocab + shares - 1) / shares, 64));
}

// as_is: x and W are both read as they lie in memory.
Layout layout_of(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, int64_t top, bool backward, bool as_is) {
    Layout l = {};
    const bool wide = dtype == RSDGC_F32;
    l.few = rows <= few_rows(dtype, as_is, backward);
    l.direct = l.few && !as_is;
    l.rows = std::min(rows, backward ? kRowChunk : kRowChunkForward);
    l.ld = up(hidden, 8);
    // planes of W: what the products need, and a copy where they cannot read it (unaligned rows: rare, so in smaller pieces)
    const bool w_for_dx = !wide && !l.few && backward;
    const int64_t w_planes = l.few ? 0 : wide || w_for_dx ? 2 : 1;
    const int64_t w_room = wide || w_for_dx || hidden % 8 ? kPackBytes : kPackBytesRare;
    const int64_t w_rows = std::min(up(vocab, 256), std::max<int64_t>(256, w_room / (std::max<int64_t>(1, w_planes) * l.ld * 2) / 256 * 256));
    const int64_t d_planes = l.few ? 3 : 2;
    const int64_t d_cols = std::min({up(vocab, 256), kMaxPiece, std::max<int64_t>(256, kPieceBytes / (std::max<int64_t>(1, l.rows) * d_planes * 2) / 256 * 256)});
    l.piece = l.few || (as_is && !w_for_dx) ? up(vocab, 256) : w_rows;
    if (backward) l.piece = std::min(l.piece, d_cols);
    l.stats_tile = l.direct ? kTile64 : choose(vocab, std::max<int64_t>(1, l.rows), hidden, 1).tile;      // direct: strips of 32 too
    l.strips = static_cast<int32_t>((vocab + kStripOf[l.stats_tile] - 1) / kStripOf[l.stats_tile]);
    if (!backward && !l.direct) {
        const int64_t side = kSide[l.stats_tile], across = (std::max<int64_t>(1, l.rows) + side - 1) / side;
        l.piece = std::min(l.piece, std::max<int64_t>(256, kMaxTiles / across * side / 256 * 256));
    }
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t here = at; at += static_cast<size_t>(up(bytes, 256)); return here; };
    l.shifts = take(kShifts * 4);
    l.parts_x = take(kMaxParts * 4);
    l.parts_w = take(kMaxParts * 4);
    l.shift_rows = take(l.rows * 4);
    if (!backward) {
        l.stats = take(l.rows * l.strips * 8);
        l.picked = take(l.rows * std::max<int64_t>(1, top) * 4);
    } else {
        if (top > 0) {
            l.idx = take(rows * top * 4);
            l.q = take(rows * top * 4);
        }
        l.gain = take(rows * 4);
        l.d_plane = l.rows * d_cols;
        l.d = take(d_planes * l.d_plane * 2);
        // shares for at least 512 workgroups, as far as the tiles alone do not give them
        const int64_t down = l.few ? 64 : 256, along = l.few && !wide_dx(dtype, rows, hidden) ? 64 : 256;
        const int64_t tiles = std::max<int64_t>(1, ((l.rows + down - 1) / down) * ((hidden + along - 1) / along));
        l.splits_most = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(64, 512 / tiles)));
        int64_t sums = l.splits_most > 1 ? 1 + l.splits_most : 1;
        if (l.direct) {
            l.share = few_share(rows, hidden, std::min(vocab, l.piece));
            sums = 1 + (std::min(vocab, l.piece) + l.share - 1) / l.share;
        }
        l.sum = take(l.rows * hidden * 4 * sums);
    }
    l.x_plane = up(l.rows * l.ld, 128);
    l.x = take((wide ? (l.few ? 3 : 2) : 1) * l.x_plane * 2);
    // x for the logits apart from x for dW: bfloat16 rows that cannot be read as they are; float32 planes by row
    if (!wide || (backward && !l.few)) l.x_raw = take((wide ? 2 : 1) * l.x_plane * 2);
    l.w_plane = up(w_rows * l.ld, 128);
    l.w = take(w_planes * l.w_plane * 2);
    l.total = std::max<size_t>(256, at);
    return l;
}

struct Call {
    int32_t dtype;
    int64_t rows, hidden, vocab;
    const void *x;
    int64_t ldx;
    const void *w;
    int64_t ldw;
    int32_t top;                       // 0: one target a row
    const int32_t *idx;
    const float *logit;
    float t;
    float *loss;
    float *lse_out;
    const float *lse, *row_grad;
    void *dx;
    int64_t lddx;
    float *dw;
    int accumulate;
    char *ws;
    hipStream_t stream;
};
template <typename T>
T *in_ws(const Call &c, size_t off) { return reinterpret_cast<T *>(c.ws + off); }

// Loads of 16 bytes where every row allows them, else of one element.
bool rows_in_16(const void *p, int64_t ld, int64_t cols, size_t size) {
    const int64_t vec = static_cast<int64_t>(16 / size);
    return aligned_to(p, 16) && ld % vec == 0 && cols % vec == 0;
}
// bfloat16 rows that the loads to LDS can take as they are
bool takes_as_is(int32_t dtype, const void *p, int64_t ld, int64_t hidden) { return dtype == RSDGC_BF16 && rows_in_16(p, ld, hidden, 2); }
Answers answers_of(const Call &c, const Layout &l, int64_t first_row) {
    Answers a = {};
    a.vocab = static_cast<int32_t>(c.vocab);
    if (c.top == 0) {
        a.idx = c.idx + first_row;
        a.top = 1;
    } else {
        a.idx = in_ws<int32_t>(c, l.idx) + first_row * c.top;
        a.q = in_ws<float>(c, l.q) + first_row * c.top;
        a.top = c.top;
    }
    return a;
}
Picked picked_by(const Call &c, const Layout &l, int64_t first_row, int64_t first) {
    const bool one = c.top == 0;
    return {one ? c.idx + first_row : nullptr, one ? nullptr : c.idx + first_row * c.top, c.top, in_ws<float>(c, l.picked), static_cast<int32_t>(first)};
}
Teacher teacher_of(const Call &c, int64_t first_row) {
    return {c.idx + first_row * c.top, c.logit + first_row * c.top, c.top, static_cast<int32_t>(c.vocab), 1.0f / c.t};
}
constexpr int64_t kAnswerBlocks = int64_t(1) << 20;      // a launch has less than 2^32 threads
size_t answer_room(const Call &c) { return static_cast<size_t>(c.top) * 32; }      // LDS of four waves
void launch_answers(const Call &c, const Layout &l) {
    hipLaunchKernelGGL(k_answers, dim3(blocks_for((c.rows + 3) / 4, kAnswerBlocks)), dim3(256), answer_room(c), c.stream, teacher_of(c, 0), c.rows, in_ws<int32_t>(c, l.idx),
                       in_ws<float>(c, l.q), c.row_grad, c.t, in_ws<float>(c, l.gain));
}

// Few rows: x's rows as bfloat16 planes.  gains: rows without an answer come out as zeros; behind a teacher its answers and the
// gains are formed on the way.
template <typename T>
void lay_few(const Call &c, const Layout &l, const Gains *gains) {
    const int cols = static_cast<int>(c.hidden), ld = static_cast<int>(l.ld);
    const Plain<T> a = {static_cast<const T *>(c.x), c.rows, c.ldx, in_ws<uint16_t>(c, l.x), l.x_plane, gains ? *gains : Gains{}, gains != nullptr, 0};
    if (gains && c.top)
        hipLaunchKernelGGL((k_plain_taught<T>), dim3(static_cast<unsigned>((c.rows + 3) / 4)), dim3(256), answer_room(c), c.stream, a, cols, ld, teacher_of(c, 0),
                           in_ws<int32_t>(c, l.idx), in_ws<float>(c, l.q), c.row_grad, c.t, in_ws<float>(c, l.gain));
    else
        hipLaunchKernelGGL((k_plain<T>), dim3(blocks_for((c.rows * l.ld / 8 + 255) / 256, 512)), dim3(256), 0, c.stream, a, cols, ld);
}
// Many rows: a matrix as float16 planes with one scale (lo may be NULL).
template <typename T>
void lay_many(const Call &c, const Layout &l, const T *w, int64_t count, uint16_t *hi, uint16_t *lo) {
    const int64_t chunks = count * l.ld / 8;
    const unsigned g = blocks_for((chunks + 255) / 256, kMaxParts), more = blocks_for((chunks + 255) / 256, kPlaneBlocks);
    float *parts = in_ws<float>(c, l.parts_w);
    const int cols = static_cast<int>(c.hidden), ld = static_cast<int>(l.ld);
    const float *every_row = nullptr;
    hipLaunchKernelGGL((k_largest<T>), dim3(g), dim3(256), 0, c.stream, w, count, cols, c.ldw, parts);
    hipLaunchKernelGGL((k_planes<T>), dim3(more), dim3(256), 0, c.stream, w, count, cols, c.ldw, every_row, parts, static_cast<int>(g), in_ws<int32_t>(c, l.shifts) + kShiftW, hi, lo, ld);
}
void align_rows(const Call &c, const Layout &l, const void *x, int64_t rows, int64_t ld, uint16_t *out) {
    hipLaunchKernelGGL(k_align, dim3(blocks_for(rows, kPlaneBlocks)), dim3(256), 0, c.stream, static_cast<const bf16 *>(x), rows, static_cast<int>(c.hidden), ld, out,
                       static_cast<int>(l.ld));
}
Operand operand(const void *base, int64_t ld, int64_t plane) {
    Operand o = {};
    o.base = static_cast<const uint16_t *>(base);
    o.ld = ld;
    o.plane = plane;
    return o;
}

// PLANES: of x and W.
template <typename T, typename V, int PLANES>
void launch_stats(const Call &c, const Layout &l, int64_t first_row, int64_t rows) {
    const bool wide = c.dtype == RSDGC_F32, x_as_is = takes_as_is(c.dtype, c.x, c.ldx, c.hidden), w_as_is = takes_as_is(c.dtype, c.w, c.ldw, c.hidden);
    const T *x = static_cast<const T *>(c.x) + first_row * c.ldx;
    uint16_t *xs = in_ws<uint16_t>(c, l.x), *ws = in_ws<uint16_t>(c, l.w);
    if (wide)
        hipLaunchKernelGGL(k_planes_by_row, dim3(static_cast<unsigned>(rows)), dim3(256), 0, c.stream, reinterpret_cast<const float *>(x), static_cast<int>(c.hidden), c.ldx,
                           in_ws<int32_t>(c, l.shift_rows), xs, xs + l.x_plane, static_cast<int>(l.ld));
    else if (!x_as_is) align_rows(c, l, x, rows, c.ldx, xs);
    const Operand xo = x_as_is ? operand(x, c.ldx, 0) : operand(xs, l.ld, l.x_plane);
    for (int64_t first = 0; first < c.vocab; first += l.piece) {
        const int64_t count = std::min(l.piece, c.vocab - first);
        const T *w = static_cast<const T *>(c.w) + first * c.ldw;
        if (wide) lay_many<T>(c, l, w, count, ws, ws + l.w_plane);
        else if (!w_as_is) align_rows(c, l, w, count, c.ldw, ws);
        const Operand wo = w_as_is ? operand(w, c.ldw, 0) : operand(ws, l.ld, l.w_plane);
        Problem p = problem(wo, xo, count, rows, c.hidden);
        const StatsArgs e = {wide ? in_ws<int32_t>(c, l.shift_rows) : nullptr, wide ? in_ws<int32_t>(c, l.shifts) + kShiftW : nullptr, 1.0f / c.t, in_ws<float2>(c, l.stats), l.strips,
                             static_cast<int32_t>(first / kStripOf[l.stats_tile]), picked_by(c, l, first_row, first)};
        with_shape<V, false, false, false, PLANES, PLANES>(l.stats_tile, [&](auto shape) {
            using S = decltype(shape);
            const dim3 grid = cut<S>(p, 1);
            hipLaunchKernelGGL((k_stats<S>), grid, dim3(S::kThreads), 0, c.stream, p, e);
        });
    }
}

void launch_loss(const Call &c, const Layout &l, int64_t first_row, int64_t rows) {
    const int vocab = static_cast<int>(c.vocab);
    const dim3 grid(static_cast<unsigned>((rows + 3) / 4));
    const float2 *stats = in_ws<float2>(c, l.stats);
    const float *picked = in_ws<float>(c, l.picked);
    float *loss = c.loss + first_row, *lse = c.lse_out + first_row;
    if (c.top) hipLaunchKernelGGL((k_loss<true>), grid, dim3(256), 2 * answer_room(c), c.stream, rows, stats, l.strips, static_cast<const int32_t *>(nullptr), picked, vocab, teacher_of(c, first_row), c.t, loss, lse);
    else hipLaunchKernelGGL((k_loss<false>), grid, dim3(256), 0, c.stream, rows, stats, l.strips, c.idx + first_row, picked, vocab, Teacher{}, c.t, loss, lse);
}

template <class S, int PLANES>
void launch_grad(const Call &c, Problem &p, const GradArgs &e, const float *gain) {
    const dim3 grid = cut<S>(p, 1), threads(S::kThreads);
    constexpr Answer kSeveral = (4 * S::TM + S::TM * S::TN) * 4 <= S::kLds ? kSpread : kLater;
    if (!c.top) hipLaunchKernelGGL((k_grad<S, PLANES, kTarget>), grid, threads, 0, c.stream, p, e);
    else hipLaunchKernelGGL((k_grad<S, PLANES, kSeveral>), grid, threads, 0, c.stream, p, e);
    if (c.top && kSeveral == kLater)
        hipLaunchKernelGGL((k_subtract<PLANES>), dim3(static_cast<unsigned>((static_cast<int64_t>(p.m) * e.answers.top + 255) / 256)), dim3(256), 0, c.stream, e.answers, gain,
                           e.many, static_cast<int64_t>(p.m), e.first, p.n, e.d, e.plane, e.ld);
}

template <typename T>
void launch_input_grad_sum(const Call &c, const InputGradArgs &e, int rows, int hidden, int splits) {
    const int64_t elements = static_cast<int64_t>(rows) * hidden;
    if (splits >= 8) hipLaunchKernelGGL((k_input_grad_sum<T, true>), dim3(static_cast<unsigned>((elements + 63) / 64)), dim3(256), 0, c.stream, e, rows, hidden, splits);
    else hipLaunchKernelGGL((k_input_grad_sum<T, false>), dim3(static_cast<unsigned>((elements + 255) / 256)), dim3(256), 0, c.stream, e, rows, hidden, splits);
}

// ---- few rows
template <typename T>
void launch_thin_weight(const Call &c, ThinWeight<T> a) {
    a.across = 32;
    while (a.across < 256 && a.across * 4 < a.hidden) a.across *= 2;
    const dim3 grid(static_cast<unsigned>((a.vocab + kThinStretch - 1) / kThinStretch), static_cast<unsigned>((a.hidden + a.across * 4 - 1) / (a.across * 4)));
    const bool whole = a.hidden % 4 == 0 && aligned_to(a.dw, 16);
    auto go = [&](auto rows) {
        if (whole) hipLaunchKernelGGL((k_thin_weight<T, rows(), true>), grid, dim3(256), 0, c.stream, a);
        else hipLaunchKernelGGL((k_thin_weight<T, rows(), false>), grid, dim3(256), 0, c.stream, a);
    };
    if (a.rows <= 4) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, kThin>{});
}
// ---- few rows, W straight from memory
template <typename T, Purpose FOR>
void launch_few_logits(const Call &c, const Layout &l, int64_t first, int64_t count, FewLogits<T> e) {
    e.w = static_cast<const T *>(c.w) + first * c.ldw;
    e.ldw = c.ldw;
    e.inv_t = 1.0f / c.t;
    const Operand none = {};
    Problem p = problem(none, operand(in_ws<uint16_t>(c, l.x), l.ld, l.x_plane), count, c.rows, c.hidden);
    const int across = c.rows <= 32 ? 32 : c.rows <= 64 ? 64 : 128;
    p.n_tiles = (p.n + across - 1) / across;
    p.splits = 1;
    auto go = [&](auto blocks, auto share) {
        p.m_tiles = (p.m + 128 / share() - 1) / (128 / share());
        hipLaunchKernelGGL((k_few_logits<T, blocks(), share(), FOR>), dim3(static_cast<unsigned>(p.m_tiles) * p.n_tiles), dim3(256), 0, c.stream, p, e);
    };
    using std::integral_constant;
    // The waves share the k axis where tiles are few and the axis is long.  The loss, or both passes, us, shared / side by side: 60 tiles
    // 6891 wide 297 / 533, 140 tiles 5132 wide 62 / 68, 225 tiles 3220 wide 596 / 547, 192 tiles 109 wide 160 / 123, 16 tiles 464 wide 20 / 30.
    const bool share = (count + 127) / 128 * p.n_tiles < 192 && c.hidden >= 384;
    if (across == 32 && share) go(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    else if (across == 32) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    else if (across == 64 && share) go(integral_constant<int, 2>{}, integral_constant<int, 4>{});
    else if (across == 64) go(integral_constant<int, 2>{}, integral_constant<int, 1>{});
    else if (share) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
}
template <typename T>
void launch_few_stats(const Call &c, const Layout &l) {
    lay_few<T>(c, l, nullptr);
    FewLogits<T> e = {};
    e.stats = in_ws<float2>(c, l.stats);
    e.strips = l.strips;
    e.picked = picked_by(c, l, 0, 0);
    if (c.top) launch_few_logits<T, kTaught>(c, l, 0, c.vocab, e);
    else launch_few_logits<T, kStats>(c, l, 0, c.vocab, e);
}
template <typename T>
void launch_few_grad(const Call &c, const Layout &l, int64_t first, int64_t count, const Gains &gains, const Answers &answers) {
    FewLogits<T> e = {};
    e.lse = c.lse;
    e.gains = gains;
    e.answers = answers;
    e.first = static_cast<int32_t>(first);
    e.d = in_ws<uint16_t>(c, l.d);
    e.plane = l.d_plane;
    e.ld = static_cast<int32_t>(l.piece);
    if (c.top) launch_few_logits<T, kMore>(c, l, first, count, e);
    else launch_few_logits<T, kOne>(c, l, first, count, e);
}
template <typename T>
void launch_few_input(const Call &c, const Layout &l, int64_t first, int64_t count, const InputGradArgs &e) {
    const int rows = static_cast<int>(c.rows), hidden = static_cast<int>(c.hidden);
    FewInput<T> a = {static_cast<const T *>(c.w) + first * c.ldw, c.ldw, in_ws<uint16_t>(c, l.d), l.d_plane, static_cast<int32_t>(l.piece), rows, hidden,
                           static_cast<int32_t>(count), l.share, in_ws<float>(c, l.sum), Problem{}, (hidden + 127) / 128};
    const int shares = static_cast<int>((count + l.share - 1) / l.share);
    a.p.m_tiles = a.across * shares;
    const int group = rows <= 32 || hidden < 4 ? 32 : 64;
    a.p.n_tiles = (rows + group - 1) / group;
    a.p.splits = 1;
    const dim3 grid(static_cast<unsigned>(a.p.m_tiles) * a.p.n_tiles);
    if (hidden < 4) hipLaunchKernelGGL((k_few_input<T, 1, true>), grid, dim3(256), 0, c.stream, a);
    else if (group == 32) hipLaunchKernelGGL((k_few_input<T, 1, false>), grid, dim3(256), 0, c.stream, a);
    else hipLaunchKernelGGL((k_few_input<T, 2, false>), grid, dim3(256), 0, c.stream, a);
    launch_input_grad_sum<T>(c, e, rows, hidden, shares);
}

// ---- dW of 9 to 128 rows (more: no registers for x).  Both passes, 32768 x 2048, us, this / tiles of 64 x 64: bfloat16 33 rows
// 162 / 205, 64 rows 183 / 217, 128 rows 255 / 289; float32 33 rows 327 / 349, 128 rows 491 / 529.
constexpr int64_t kFewWeight = 128;
template <typename T>
void launch_few_weight(const Call &c, const Operand &d, int64_t count, const FewWeight<T> &of) {
    Problem p = problem(d, Operand{}, count, c.hidden, c.rows);
    FewWeight<T> e = of;
    auto go = [&](auto steps, auto columns) {
        const int64_t across = (c.hidden + 128 * columns() - 1) / (128 * columns());
        e.stretch = static_cast<int32_t>(up(std::max<int64_t>(1, count * across / 768), 64));
        hipLaunchKernelGGL((k_few_weight<T, steps(), columns()>), dim3(static_cast<unsigned>((count + e.stretch - 1) / e.stretch), static_cast<unsigned>(across)), dim3(256), 0,
                           c.stream, p, e);
    };
    using std::integral_constant;
    constexpr bool kWide = sizeof(T) == 4;
    if (c.rows <= 32) go(integral_constant<int, 2>{}, integral_constant<int, 4>{});
    else if (c.rows <= 64) go(integral_constant<int, 4>{}, integral_constant<int, kWide ? 2 : 4>{});
    else go(integral_constant<int, 8>{}, integral_constant<int, kWide ? 1 : 2>{});
}

// V: type of the logits' operands, PLANES: of these; D: type of d's planes, D_PLANES: of these.
template <typename T, typename V, int PLANES, typename D, int D_PLANES>
void launch_backward(const Call &c, const Layout &l, int64_t first_row, int64_t rows, bool accumulate) {
    const bool wide = c.dtype == RSDGC_F32, few = l.few, x_as_is = takes_as_is(c.dtype, c.x, c.ldx, c.hidden), w_as_is = takes_as_is(c.dtype, c.w, c.ldw, c.hidden);
    const int cols = static_cast<int>(c.hidden), ld = static_cast<int>(l.ld);
    const T *x = static_cast<const T *>(c.x) + first_row * c.ldx;
    float *parts = in_ws<float>(c, l.parts_x), *gain = in_ws<float>(c, l.gain) + first_row;
    int32_t *shifts = in_ws<int32_t>(c, l.shifts), *shift_rows = in_ws<int32_t>(c, l.shift_rows);
    uint16_t *xs = in_ws<uint16_t>(c, l.x), *x_raw = in_ws<uint16_t>(c, l.x_raw), *ws = in_ws<uint16_t>(c, l.w), *d = in_ws<uint16_t>(c, l.d);
    const Answers a = answers_of(c, l, first_row);
    const Gains gains = few && !c.top ? Gains{nullptr, c.row_grad + first_row, a.idx, a.vocab} : Gains{gain, nullptr, nullptr, 0};
    if (!few) {
        const unsigned g = blocks_for(rows, kMaxParts), more = blocks_for((rows * l.ld / 8 + 255) / 256, kPlaneBlocks);
        uint16_t *second = wide ? xs + l.x_plane : nullptr;
        hipLaunchKernelGGL((k_gain<T>), dim3(g), dim3(256), 0, c.stream, a, c.row_grad + first_row, c.t, x, rows, cols, c.ldx, gain, parts, shift_rows, x_raw, x_raw + l.x_plane, ld);
        hipLaunchKernelGGL((k_planes<T>), dim3(more), dim3(256), 0, c.stream, x, rows, cols, c.ldx, gain, parts, static_cast<int>(g), shifts + kShiftX, xs, second, ld);
        if (!wide && !x_as_is) align_rows(c, l, x, rows, c.ldx, x_raw);
    }
    // for the logits: as it is, planes under a scale by row (float32), or the copy (few rows: without the rows that have no answer)
    const Operand xo = x_as_is ? operand(x, c.ldx, 0) : few ? operand(xs, l.ld, l.x_plane) : operand(x_raw, l.ld, l.x_plane);
    const Operand x_planes = operand(xs, l.ld, l.x_plane);
    for (int64_t first = 0; first < c.vocab; first += l.piece) {
        const int64_t count = std::min(l.piece, c.vocab - first);
        const int32_t ldd = static_cast<int32_t>(l.piece);
        const T *w = static_cast<const T *>(c.w) + first * c.ldw;
        // x's copy (few rows) also serves dW's product; a teacher's answers are formed with it
        if (few) {
            if (first == 0 && (l.direct || c.top || rows > kThin)) lay_few<T>(c, l, &gains);
        } else if (wide) lay_many<T>(c, l, w, count, ws, ws + l.w_plane);
        else if (!w_as_is) align_rows(c, l, w, count, c.ldw, ws);
        const Operand wo = w_as_is ? operand(w, c.ldw, 0) : operand(ws, l.ld, l.w_plane), d_planes = operand(d, ldd, l.d_plane);
        if (l.direct) launch_few_grad<T>(c, l, first, count, gains, a);
        else if constexpr (PLANES < 3) {
            Problem p = problem(xo, wo, rows, count, c.hidden);
            const GradArgs e = {!few, wide ? shift_rows : nullptr, wide ? shifts + kShiftW : nullptr, 1.0f / c.t, c.lse + first_row, gains, a, static_cast<int32_t>(first), d, l.d_plane, ldd};
            with_shape<V, false, false, true, PLANES, PLANES>(choose(rows, count, c.hidden, 1).tile,
                                                              [&](auto shape) { launch_grad<decltype(shape), D_PLANES>(c, p, e, gain); });
        }
        const InputGradArgs dx = {few ? nullptr : shifts + kShiftW, gains, first == 0, first + count == c.vocab, in_ws<float>(c, l.sum), static_cast<T *>(c.dx) + first_row * c.lddx, c.lddx};
        if (l.direct) launch_few_input<T>(c, l, first, count, dx);
        else if constexpr (PLANES < 3) {
            Operand wd = wo;
            if (!wide && !few) {
                wd = operand(ws + l.w_plane, l.ld, 0);
                lay_many<T>(c, l, w, count, ws + l.w_plane, nullptr);
            }
            Problem p = problem(d_planes, wd, rows, c.hidden, count);
            Choice how = choose(rows, c.hidden, count, l.splits_most);
            if (wide_dx(c.dtype, c.rows, c.hidden)) how = {kTileWide, std::max<int64_t>(1, std::min<int64_t>(l.splits_most, 512 / ((c.hidden + 255) / 256)))};
            constexpr int kForDx = D_PLANES == 3 ? 2 : D_PLANES;      // bfloat16, few rows: two planes of d are good to 2^-18, a float32 sum's error
            with_shape<D, false, true, false, kForDx, PLANES>(how.tile, [&](auto shape) {
                using S = decltype(shape);
                const dim3 grid = cut<S>(p, how.splits);
                hipLaunchKernelGGL((k_input_grad<S, T>), grid, dim3(S::kThreads), 0, c.stream, p, dx);
            });
            if (p.splits > 1) launch_input_grad_sum<T>(c, dx, p.m, p.n, p.splits);
        }
        if (few && rows <= kThin) {         // a last chunk of many rows may be as short, with two scaled planes of d
            launch_thin_weight<T>(c, {x, c.ldx, gains, static_cast<int32_t>(rows), cols, static_cast<int32_t>(count), d, l.d_plane, ldd, c.dw + first * c.hidden, accumulate, 0});
        } else if (few && rows <= kFewWeight) {
            launch_few_weight<T>(c, d_planes, count, {x, c.ldx, gains, c.dw + first * c.hidden, accumulate, 0});
        } else {
            Problem p = problem(d_planes, x_planes, count, c.hidden, rows);
            const WeightGradArgs e = {few ? nullptr : shifts + kShiftX, c.dw + first * c.hidden, accumulate};
            with_shape<D, true, true, false, D_PLANES, PLANES>(choose(count, c.hidden, rows, 1, D_PLANES == 3 ? kTile64 : kTile256).tile, [&](auto shape) {
                using S = decltype(shape);
                const dim3 grid = cut<S>(p, 1);
                hipLaunchKernelGGL((k_weight_grad<S>), grid, dim3(S::kThreads), 0, c.stream, p, e);
            });
        }
    }
}

// ---- arguments
bool sizes_ok(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab) {
    return type_known(dtype) && rows >= 0 && rows <= kMaxRows && hidden >= 1 && hidden <= kMaxStride && vocab >= 1 && vocab <= kMaxVocab;
}
// What a call writes may touch nothing else that it reads or writes.
bool apart(const Range *written, int n_written, const Range *read, int n_read) {
    for (int i = 0; i < n_written; ++i) {
        for (int j = i + 1; j < n_written; ++j)
            if (ranges_overlap(written[i], written[j])) return false;
        for (int j = 0; j < n_read; ++j)
            if (ranges_overlap(written[i], read[j])) return false;
    }
    return true;
}

bool inputs_ok(const Call &c) {
    const size_t size = type_size(c.dtype);
    if (!sizes_ok(c.dtype, c.rows, c.hidden, c.vocab) || c.ldx < c.hidden || c.ldw < c.hidden || c.ldx > kMaxStride || c.ldw > kMaxStride) return false;
    if (c.top < 0 || c.top > RSDGC_MAX_TOP || !std::isfinite(c.t) || !(c.t > 0.0f) || !std::isfinite(1.0f / c.t)) return false;
    if (!c.w || !aligned_to(c.w, size) || !c.ws || !aligned_to(c.ws, 256)) return false;
    if (c.rows == 0) return true;
    return c.x && aligned_to(c.x, size) && c.idx && aligned_to(c.idx, 4) && (c.top == 0 || (c.logit && aligned_to(c.logit, 4)));
}
void read_by(const Call &c, Range (&r)[4]) {
    const size_t size = type_size(c.dtype), entries = static_cast<size_t>(c.rows) * std::max(1, c.top) * 4;
    r[0] = matrix_range(c.x, c.rows, c.hidden, c.ldx, size);
    r[1] = matrix_range(c.w, c.vocab, c.hidden, c.ldw, size);
    r[2] = {c.idx, entries};
    r[3] = {c.logit, c.top ? entries : 0};
}
// Whether x and W are both read as they lie in memory.
bool as_is(const Call &c) { return takes_as_is(c.dtype, c.x, c.ldx, c.hidden) && takes_as_is(c.dtype, c.w, c.ldw, c.hidden); }

int forward(const Call &c, const char *what) {
    if (!inputs_ok(c)) return RSDGC_EINVAL;
    if (c.rows == 0) return RSDGC_OK;
    if (!c.loss || !c.lse_out || !aligned_to(c.loss, 4) || !aligned_to(c.lse_out, 4)) return RSDGC_EINVAL;
    const Layout l = layout_of(c.dtype, c.rows, c.hidden, c.vocab, c.top, false, as_is(c));
    const Range written[] = {{c.loss, static_cast<size_t>(c.rows) * 4}, {c.lse_out, static_cast<size_t>(c.rows) * 4}, {c.ws, l.total}};
    Range read[4];
    read_by(c, read);
    if (!apart(written, 3, read, 4)) return RSDGC_EINVAL;
    for (int64_t first = 0; first < c.rows; first += l.rows) {
        const int64_t rows = std::min(l.rows, c.rows - first);
        if (c.dtype == RSDGC_BF16) {
            if (l.direct) launch_few_stats<bf16>(c, l);
            else launch_stats<bf16, bfloat8, 1>(c, l, first, rows);
        } else {
            if (l.direct) launch_few_stats<float>(c, l);
            else launch_stats<float, half8, 2>(c, l, first, rows);
        }
        launch_loss(c, l, first, rows);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? RSDGC_OK : remember_hip_error(e, what);
}

int backward(const Call &c, const char *what) {
    if (!inputs_ok(c) || !c.dw || !aligned_to(c.dw, 4)) return RSDGC_EINVAL;
    const size_t size = type_size(c.dtype);
    if (c.rows > 0 && (!c.lse || !c.row_grad || !c.dx || c.lddx < c.hidden || c.lddx > kMaxStride || !aligned_to(c.lse, 4) || !aligned_to(c.row_grad, 4) || !aligned_to(c.dx, size))) return RSDGC_EINVAL;
    const Layout l = layout_of(c.dtype, c.rows, c.hidden, c.vocab, c.top, true, as_is(c));
    Range read[6];
    Range (&four)[4] = *reinterpret_cast<Range (*)[4]>(read);
    read_by(c, four);
    read[4] = {c.lse, static_cast<size_t>(c.rows) * 4};
    read[5] = {c.row_grad, static_cast<size_t>(c.rows) * 4};
    const Range written[] = {matrix_range(c.dx, c.rows, c.hidden, c.lddx, size), {c.dw, static_cast<size_t>(c.vocab) * c.hidden * 4}, {c.ws, l.total}};
    if (!apart(written, 3, read, 6)) return RSDGC_EINVAL;
    if (c.rows == 0) {
        if (!c.accumulate) hipLaunchKernelGGL(k_clear, dim3(1024), dim3(256), 0, c.stream, c.dw, c.vocab * c.hidden);
    } else {
        if (c.top && !l.few) launch_answers(c, l);
        for (int64_t first = 0; first < c.rows; first += l.rows) {
            const int64_t rows = std::min(l.rows, c.rows - first);
            const bool accumulate = c.accumulate || first > 0;
            if (c.dtype == RSDGC_BF16) {
                if (l.few) launch_backward<bf16, bfloat8, 1, bfloat8, 3>(c, l, first, rows, accumulate);
                else launch_backward<bf16, bfloat8, 1, half8, 2>(c, l, first, rows, accumulate);
            } else {
                if (l.few) launch_backward<float, bfloat8, 3, bfloat8, 3>(c, l, first, rows, accumulate);
                else launch_backward<float, half8, 2, half8, 2>(c, l, first, rows, accumulate);
            }
        }
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? RSDGC_OK : remember_hip_error(e, what);
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" {

size_t rsdgc_head_workspace_bytes(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, int32_t top, int backward) {
    if (!sizes_ok(dtype, rows, hidden, vocab) || top < 0 || top > RSDGC_MAX_TOP) return 0;
    // whichever way the operands will lie in memory
    auto of = [&](bool with_gradients) {
        return std::max(layout_of(dtype, rows, hidden, vocab, top, with_gradients, false).total, layout_of(dtype, rows, hidden, vocab, top, with_gradients, true).total);
    };
    return backward ? std::max(of(false), of(true)) : of(false);
}

int rsdgc_head_loss(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, const void *x, int64_t ldx, const void *w, int64_t ldw,
                    const int32_t *target, float *loss, float *lse, void *workspace, void *stream) {
    Call c = {};
    c.dtype = dtype; c.rows = rows; c.hidden = hidden; c.vocab = vocab;
    c.x = x; c.ldx = ldx; c.w = w; c.ldw = ldw;
    c.idx = target; c.t = 1.0f;
    c.loss = loss; c.lse_out = lse;
    c.ws = static_cast<char *>(workspace); c.stream = static_cast<hipStream_t>(stream);
    return forward(c, "rsdgc_head_loss");
}

int rsdgc_head_loss_backward(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, const void *x, int64_t ldx, const void *w,
                             int64_t ldw, const int32_t *target, const float *lse, const float *row_grad, void *dx, int64_t lddx,
                             float *dw, int accumulate, void *workspace, void *stream) {
    Call c = {};
    c.dtype = dtype; c.rows = rows; c.hidden = hidden; c.vocab = vocab;
    c.x = x; c.ldx = ldx; c.w = w; c.ldw = ldw;
    c.idx = target; c.t = 1.0f;
    c.lse = lse; c.row_grad = row_grad; c.dx = dx; c.lddx = lddx; c.dw = dw; c.accumulate = accumulate != 0;
    c.ws = static_cast<char *>(workspace); c.stream = static_cast<hipStream_t>(stream);
    return backward(c, "rsdgc_head_loss_backward");
}

int rsdgc_distill_loss(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, const void *x, int64_t ldx, const void *w, int64_t ldw,
                       int32_t top, const int32_t *top_idx, const float *top_logit, double temperature, float *loss, float *lse,
                       void *workspace, void *stream) {
    if (top < 1) return RSDGC_EINVAL;
    Call c = {};
    c.dtype = dtype; c.rows = rows; c.hidden = hidden; c.vocab = vocab;
    c.x = x; c.ldx = ldx; c.w = w; c.ldw = ldw;
    c.top = top; c.idx = top_idx; c.logit = top_logit; c.t = static_cast<float>(temperature);
    c.loss = loss; c.lse_out = lse;
    c.ws = static_cast<char *>(workspace); c.stream = static_cast<hipStream_t>(stream);
    return forward(c, "rsdgc_distill_loss");
}

int rsdgc_distill_loss_backward(int32_t dtype, int64_t rows, int64_t hidden, int64_t vocab, const void *x, int64_t ldx, const void *w,
                                int64_t ldw, int32_t top, const int32_t *top_idx, const float *top_logit, double temperature,
                                const float *lse, const float *row_grad, void *dx, int64_t lddx, float *dw, int accumulate,
                                void *workspace, void *stream) {
    if (top < 1) return RSDGC_EINVAL;
    Call c = {};
    c.dtype = dtype; c.rows = rows; c.hidden = hidden; c.vocab = vocab;
    c.x = x; c.ldx = ldx; c.w = w; c.ldw = ldw;
    c.top = top; c.idx = top_idx; c.logit = top_logit; c.t = static_cast<float>(temperature);
    c.lse = lse; c.row_grad = row_grad; c.dx = dx; c.lddx = lddx; c.dw = dw; c.accumulate = accumulate != 0;
    c.ws = static_cast<char *>(workspace); c.stream = static_cast<hipStream_t>(stream);
    return backward(c, "rsdgc_distill_loss_backward");
}

}  // extern "C"
