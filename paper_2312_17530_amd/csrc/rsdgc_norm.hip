// Layer normalisation, forward and backward (gfx950, wave64).
//
//   forward    mean and rstd = 1 / sqrt(var + eps) of each row, y = (x - mean) * rstd * gamma + beta
//   backward   h = dy * gamma, xh = (x - mean) * rstd:  dx = rstd * (h - mean(h) - xh * mean(h * xh)),
//              dgamma = sum over rows of dy * xh, dbeta = sum over rows of dy
//
// A row is held in the registers of the threads that share it (up to kHeld elements each), so every input is read once; the
// variance is taken around the mean, not from a difference of squares.  The sums over rows stay in the registers of the
// thread that owns the columns while its group goes from row to row; each workgroup then leaves one line of partial sums and
// a second launch adds the lines up in a fixed order.  Everything is summed in float32.
//
// Bound by memory.  Forward 65536 x 2048 bfloat16 97 us = 5.5 TB/s (read and written), backward 174 us = 4.6 TB/s and 6 us for the lines;
// 8192 x 4096 25 and 51 + 5 us; one row of 4096 3 us, a launch.  A copy of this size reaches 5.1 TB/s on this card.
#include "rsdgc_training.h"

#include <algorithm>
#include <cmath>

namespace rsdgc {
namespace {

constexpr int kHeld = 16;              // elements of a row that one thread holds
constexpr int kMaxThreads = 1024;      // that share a row in the forward pass; wider rows take other kernels
constexpr int kBackwardThreads = 512;  // ... in the backward pass, whose threads need more registers
constexpr int kGroupThreads = 512;     // threads of a backward workgroup whose rows are narrower
constexpr int kMaxLines = 512;         // lines of partial sums, two workgroups per CU
constexpr int kForwardBlocks = 2048;   // workgroups of 256 threads that go over the rows in the forward pass, eight per CU; of the wide kernels'

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Chunk { T v[VEC]; };

// Sum over the THREADS threads that share a row; `red` holds a float for every wave of the workgroup.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float *red, int group) {
    v = wave_sum(v);
    if (THREADS == 64) return v;
    constexpr int kWaves = THREADS / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();                   // the last sums have been read
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < kWaves; ++w) s += red[group * kWaves + w];
    return s;
}

template <typename T>
struct ForwardArgs {
    const T *x;
    const float *gamma, *beta;
    T *y;
    float *mean, *rstd;
    int64_t rows, ldx, ldy;
    int32_t cols;
    float eps;
};

// A row's elements as its threads hold them, zeros beyond its end and beyond the last row.
template <typename T, int VEC, int THREADS, int HELD>
struct RowHeld {
    Chunk<T, VEC> q[HELD / VEC];
    __device__ __forceinline__ void load(const T *x, int64_t ld, int64_t row, int64_t rows, int cols, int t) {
        const T *from = x + (row < rows ? row : 0) * ld;
#pragma unroll
        for (int i = 0; i < HELD / VEC; ++i) {
            const int c = (i * THREADS + t) * VEC;
            if (row < rows && c < cols) q[i] = *reinterpret_cast<const Chunk<T, VEC> *>(from + c);
            else q[i] = Chunk<T, VEC>{};
        }
    }
};

// cols floats (or `fill` for NULL) as the threads of a row hold its elements.
template <int VEC, int THREADS, int HELD>
__device__ __forceinline__ void load_params(const float *from, float fill, int cols, int t, float (&to)[HELD / VEC][VEC]) {
#pragma unroll
    for (int i = 0; i < HELD / VEC; ++i) {
        const int c = (i * THREADS + t) * VEC;
        if (from && c < cols) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) to[i][e] = from[c + e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) to[i][e] = c < cols ? fill : 0.0f;
        }
    }
}

// THREADS threads per row, the workgroup's groups side by side; VEC elements per load.  A workgroup goes from row to row with
// the scale and the shift in its registers.
template <typename T, int VEC, int THREADS, int GROUPS>
__global__ __launch_bounds__(THREADS * GROUPS) void k_norm_forward(const ForwardArgs<T> a) {
    __shared__ float red[THREADS * GROUPS / 64];
    constexpr int kParts = kHeld / VEC;
    const int group = threadIdx.x / THREADS, t = threadIdx.x % THREADS;
    float gamma[kParts][VEC], beta[kParts][VEC];
    load_params<VEC, THREADS, kHeld>(a.gamma, 1.0f, a.cols, t, gamma);
    load_params<VEC, THREADS, kHeld>(a.beta, 0.0f, a.cols, t, beta);
    const float share = 1.0f / static_cast<float>(a.cols);
    const int64_t down = static_cast<int64_t>(gridDim.x) * GROUPS;
    RowHeld<T, VEC, THREADS, kHeld> next;
    next.load(a.x, a.ldx, static_cast<int64_t>(blockIdx.x) * GROUPS + group, a.rows, a.cols, t);
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * GROUPS; first < a.rows; first += down) {
        const int64_t row = first + group;
        const bool live = row < a.rows;
        float v[kParts][VEC];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) { v[i][e] = to_float(next.q[i].v[e]); s += v[i][e]; }
        next.load(a.x, a.ldx, row + down, a.rows, a.cols, t);      // on its way while this row is summed
        const float mean = row_sum<THREADS>(s, red, group) * share;
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            if ((i * THREADS + t) * VEC < a.cols)
#pragma unroll
                for (int e = 0; e < VEC; ++e) { const float d = v[i][e] - mean; q = fmaf(d, d, q); }
        const float rstd = 1.0f / sqrtf(row_sum<THREADS>(q, red, group) * share + a.eps);
        if (!live) continue;
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T *y = a.y + row * a.ldy;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (i * THREADS + t) * VEC;
            if (c >= a.cols) break;
            Chunk<T, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; ++e) o.v[e] = static_cast<T>(fmaf((v[i][e] - mean) * rstd, gamma[i][e], beta[i][e]));
            *reinterpret_cast<Chunk<T, VEC> *>(y + c) = o;
        }
    }
}

// Rows too wide for the registers: three sweeps over the row, which lies in the cache after the first.
template <typename T>
__global__ __launch_bounds__(kMaxThreads) void k_norm_forward_wide(const ForwardArgs<T> a) {
    __shared__ float red[kMaxThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = a.x + row * a.ldx;
        float s = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kMaxThreads) s += to_float(x[c]);
        const float mean = row_sum<kMaxThreads>(s, red, 0) / static_cast<float>(a.cols);
        float q = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kMaxThreads) { const float d = to_float(x[c]) - mean; q = fmaf(d, d, q); }
        const float rstd = 1.0f / sqrtf(row_sum<kMaxThreads>(q, red, 0) / static_cast<float>(a.cols) + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T *y = a.y + row * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += kMaxThreads) {
            const float unit = (to_float(x[c]) - mean) * rstd;
            y[c] = static_cast<T>(fmaf(unit, a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f));
        }
    }
}

template <typename T>
struct BackwardArgs {
    const T *dy, *x;
    const float *gamma, *mean, *rstd;
    T *dx;
    float *lines;                      // [workgroup][2][cols]
    int64_t rows, lddy, ldx, lddx;
    int32_t cols;
};

// A workgroup takes rows blockIdx * GROUPS + group, then on by the grid.
template <typename T, int VEC, int THREADS, int GROUPS>
__global__ __launch_bounds__(THREADS * GROUPS) void k_norm_backward(const BackwardArgs<T> a) {
    __shared__ float red[2][THREADS * GROUPS / 64];
    __shared__ float fold[GROUPS > 1 ? THREADS * GROUPS * kHeld / 2 : 1];
    constexpr int kParts = kHeld / VEC, kWaves = THREADS / 64;
    const int group = threadIdx.x / THREADS, t = threadIdx.x % THREADS;
    float gamma[kParts][VEC], dg[kParts][VEC], db[kParts][VEC];
    load_params<VEC, THREADS, kHeld>(a.gamma, 1.0f, a.cols, t, gamma);
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dg[i][e] = db[i][e] = 0.0f;
    const float share = 1.0f / static_cast<float>(a.cols);
    const int64_t down = static_cast<int64_t>(gridDim.x) * GROUPS;
    RowHeld<T, VEC, THREADS, kHeld> next_x, next_dy;
    float next_mean, next_rstd;
    auto ahead = [&](int64_t row) {
        next_x.load(a.x, a.ldx, row, a.rows, a.cols, t);
        next_dy.load(a.dy, a.lddy, row, a.rows, a.cols, t);
        next_mean = row < a.rows ? a.mean[row] : 0.0f;
        next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
    };
    ahead(static_cast<int64_t>(blockIdx.x) * GROUPS + group);
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * GROUPS; first < a.rows; first += down) {
        const int64_t row = first + group;
        const bool live = row < a.rows;
        const float mean = next_mean, rstd = next_rstd;
        float g[kParts][VEC], xh[kParts][VEC];
        float sh = 0.0f, shx = 0.0f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const bool in = live && (i * THREADS + t) * VEC < a.cols;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                g[i][e] = to_float(next_dy.q[i].v[e]);
                xh[i][e] = in ? (to_float(next_x.q[i].v[e]) - mean) * rstd : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float h = g[i][e] * gamma[i][e];
                sh += h;
                shx = fmaf(h, xh[i][e], shx);
                dg[i][e] = fmaf(g[i][e], xh[i][e], dg[i][e]);
                db[i][e] += g[i][e];
            }
        }
        ahead(row + down);             // on its way while this row is summed
        sh = wave_sum(sh);
        shx = wave_sum(shx);
        if (THREADS > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = sh; red[1][threadIdx.x >> 6] = shx; }
            __syncthreads();
            sh = shx = 0.0f;
            for (int w = 0; w < kWaves; ++w) { sh += red[0][group * kWaves + w]; shx += red[1][group * kWaves + w]; }
        }
        sh *= share;
        shx *= share;
        if (live) {
            T *dx = a.dx + row * a.lddx;
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                const int c = (i * THREADS + t) * VEC;
                if (c >= a.cols) break;
                Chunk<T, VEC> o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    o.v[e] = static_cast<T>(rstd * (g[i][e] * gamma[i][e] - sh - xh[i][e] * shx));
                }
                *reinterpret_cast<Chunk<T, VEC> *>(dx + c) = o;
            }
        }
    }
    if (!a.lines) return;
    // the groups' sums, folded in halves through LDS
    if (GROUPS > 1)
        for (int half = GROUPS / 2; half; half /= 2) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
                if (group >= half && group < 2 * half)
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) fold[((group - half) * kHeld + i) * THREADS + t] = (which ? db : dg)[i / VEC][i % VEC];
                __syncthreads();
                if (group < half)
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) (which ? db : dg)[i / VEC][i % VEC] += fold[(group * kHeld + i) * THREADS + t];
            }
        }
    if (group) return;
    float *line = a.lines + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = (i * THREADS + t) * VEC + e;
            if (c < a.cols) { line[c] = dg[i][e]; line[a.cols + c] = db[i][e]; }
        }
}

// Rows too wide for the registers: two sweeps over the row for dx, and the sums over rows in a launch of their own.
template <typename T>
__global__ __launch_bounds__(kMaxThreads) void k_norm_backward_wide(const BackwardArgs<T> a) {
    __shared__ float red[kMaxThreads / 64];
    const float share = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = a.dy + row * a.lddy, *x = a.x + row * a.ldx;
        T *dx = a.dx + row * a.lddx;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sh = 0.0f, shx = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kMaxThreads) {
            const float g = to_float(dy[c]), xh = (to_float(x[c]) - mean) * rstd, h = a.gamma ? g * a.gamma[c] : g;
            sh += h;
            shx = fmaf(h, xh, shx);
        }
        sh = row_sum<kMaxThreads>(sh, red, 0) * share;
        shx = row_sum<kMaxThreads>(shx, red, 0) * share;
        for (int c = threadIdx.x; c < a.cols; c += kMaxThreads) {
            const float g = to_float(dy[c]), xh = (to_float(x[c]) - mean) * rstd, h = a.gamma ? g * a.gamma[c] : g;
            dx[c] = static_cast<T>(rstd * (h - sh - xh * shx));
        }
    }
}
// The sums of rows blockIdx.y, blockIdx.y + gridDim.y, ... for 256 columns; before k_norm_backward_wide, which may write over dy or x.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_columns(const BackwardArgs<T> a) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = to_float(a.dy[row * a.lddy + c]);
        dg = fmaf(g, (to_float(a.x[row * a.ldx + c]) - a.mean[row]) * a.rstd[row], dg);
        db += g;
    }
    float *line = a.lines + static_cast<int64_t>(blockIdx.y) * 2 * a.cols;
    line[c] = dg;
    line[a.cols + c] = db;
}

// The lines' sum: a workgroup takes 64 of the 2 * cols columns, its sixteen waves every sixteenth line.
constexpr int kLineWaves = 16;
__global__ __launch_bounds__(64 * kLineWaves) void k_norm_lines(const float *lines, int32_t n_lines, int32_t cols, float *dgamma, float *dbeta, int accumulate) {
    __shared__ float part[kLineWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + lane, width = 2 * static_cast<int64_t>(cols);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < width) {
        int l = wave;
        for (; l + 3 * kLineWaves < n_lines; l += 4 * kLineWaves)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += lines[(l + u * kLineWaves) * width + c];
        for (; l < n_lines; l += kLineWaves) s[0] += lines[l * width + c];
    }
    part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave || c >= width) return;
    float sum = 0.0f;
    for (int w = 0; w < kLineWaves; ++w) sum += part[w][lane];
    float *out = c < cols ? dgamma : dbeta;
    if (!out) return;
    const int64_t at = c < cols ? c : c - cols;
    out[at] = accumulate ? out[at] + sum : sum;
}

// ---- host side ---------------------------------------------------------------
// Rows in registers as far as they fit, else the wide kernels: 2048 rows of 16384 bfloat16 28 us forward, of 16392 59; of 8192 63 us both
// ways, of 8200 89.
int threads_per_row(int64_t cols) {
    int t = 64;
    while (static_cast<int64_t>(t) * kHeld < cols) t *= 2;
    return t;                            // over kMaxThreads: the wide kernels
}
int groups_of(int threads) { return std::max(1, kGroupThreads / threads); }
int n_lines(int64_t rows, int64_t cols) {
    const int t = threads_per_row(cols), g = t > kBackwardThreads ? 1 : groups_of(t);
    return static_cast<int>(std::min<int64_t>(kMaxLines, (rows + g - 1) / g));
}

template <typename T, int VEC, int THREADS>
void forward_of(const ForwardArgs<T> &a, hipStream_t s) {
    constexpr int kGroups = THREADS >= 256 ? 1 : 256 / THREADS;
    const int64_t blocks = std::min<int64_t>(kForwardBlocks * 256 / (THREADS * kGroups), (a.rows + kGroups - 1) / kGroups);
    hipLaunchKernelGGL((k_norm_forward<T, VEC, THREADS, kGroups>), dim3(static_cast<unsigned>(blocks)), dim3(THREADS * kGroups), 0, s, a);
}
template <typename T, int VEC>
void forward_vec(const ForwardArgs<T> &a, hipStream_t s) {
    switch (threads_per_row(a.cols)) {
        case 64: return forward_of<T, VEC, 64>(a, s);
        case 128: return forward_of<T, VEC, 128>(a, s);
        case 256: return forward_of<T, VEC, 256>(a, s);
        case 512: return forward_of<T, VEC, 512>(a, s);
        default: return forward_of<T, VEC, 1024>(a, s);
    }
}
template <typename T, int VEC, int THREADS>
void backward_of(const BackwardArgs<T> &a, int blocks, hipStream_t s) {
    constexpr int kGroups = THREADS >= kGroupThreads ? 1 : kGroupThreads / THREADS;
    hipLaunchKernelGGL((k_norm_backward<T, VEC, THREADS, kGroups>), dim3(blocks), dim3(THREADS * kGroups), 0, s, a);
}
template <typename T, int VEC>
void backward_vec(const BackwardArgs<T> &a, int blocks, hipStream_t s) {
    switch (threads_per_row(a.cols)) {
        case 64: return backward_of<T, VEC, 64>(a, blocks, s);
        case 128: return backward_of<T, VEC, 128>(a, blocks, s);
        case 256: return backward_of<T, VEC, 256>(a, blocks, s);
        default: return backward_of<T, VEC, 512>(a, blocks, s);
    }
}

// Loads of 16 bytes where every row allows them, else of one element: 8192 rows of 4096 bfloat16 23 us forward, 78 both ways, of 4095
// 27 and 88.
bool rows_in_16(const void *p, int64_t ld, int64_t cols, size_t size) {
    const int64_t vec = static_cast<int64_t>(16 / size);
    return aligned_to(p, 16) && ld % vec == 0 && cols % vec == 0;
}

template <typename T>
void forward_typed(const ForwardArgs<T> &a, hipStream_t s) {
    if (threads_per_row(a.cols) > kMaxThreads)
        hipLaunchKernelGGL((k_norm_forward_wide<T>), dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kForwardBlocks))), dim3(kMaxThreads), 0, s, a);
    else if (rows_in_16(a.x, a.ldx, a.cols, sizeof(T)) && rows_in_16(a.y, a.ldy, a.cols, sizeof(T)))
        forward_vec<T, 16 / sizeof(T)>(a, s);
    else
        forward_vec<T, 1>(a, s);
}
template <typename T>
void backward_typed(const BackwardArgs<T> &a, int blocks, hipStream_t s) {
    if (threads_per_row(a.cols) > kBackwardThreads) {
        if (a.lines) hipLaunchKernelGGL((k_norm_columns<T>), dim3(static_cast<unsigned>((a.cols + 255) / 256), blocks), dim3(256), 0, s, a);
        hipLaunchKernelGGL((k_norm_backward_wide<T>), dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kForwardBlocks))), dim3(kMaxThreads), 0, s, a);
    }
    else if (rows_in_16(a.x, a.ldx, a.cols, sizeof(T)) && rows_in_16(a.dy, a.lddy, a.cols, sizeof(T)) && rows_in_16(a.dx, a.lddx, a.cols, sizeof(T)))
        backward_vec<T, 16 / sizeof(T)>(a, blocks, s);
    else
        backward_vec<T, 1>(a, blocks, s);
}

constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int64_t kMaxCols = int64_t(1) << 24;
bool sizes_ok(int32_t dtype, int64_t rows, int64_t cols) { return type_known(dtype) && rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxCols; }

// a and b may be the same rows, or apart; not shifted against each other.
bool same_or_apart(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, int64_t cols, size_t size) {
    if (a == b && lda == ldb) return true;
    return !ranges_overlap(matrix_range(a, rows, cols, lda, size), matrix_range(b, rows, cols, ldb, size));
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" {

size_t rsdgc_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return 0;
    const size_t need = static_cast<size_t>(n_lines(rows, cols)) * 2 * static_cast<size_t>(cols) * sizeof(float);
    return std::max<size_t>(256, (need + 255) / 256 * 256);
}

int rsdgc_layer_norm(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, const float *gamma,
                     const float *beta, double eps, void *y, int64_t ldy, float *mean, float *rstd, void *stream_) {
    if (!sizes_ok(dtype, rows, cols) || ldx < cols || ldy < cols || !(eps >= 0.0) || !std::isfinite(eps)) return RSDGC_EINVAL;
    if (rows == 0) return RSDGC_OK;
    const size_t size = type_size(dtype);
    if (!x || !y || !aligned_to(x, size) || !aligned_to(y, size) || !aligned_to(gamma, 4) || !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return RSDGC_EINVAL;
    if (!same_or_apart(x, ldx, y, ldy, rows, cols, size)) return RSDGC_EINVAL;
    const size_t ny = extent_bytes(rows, cols, ldy, size), nx = extent_bytes(rows, cols, ldx, size), nc = static_cast<size_t>(cols) * 4, nr = static_cast<size_t>(rows) * 4;
    if (ranges_overlap(y, ny, gamma, nc) || ranges_overlap(y, ny, beta, nc) || ranges_overlap(y, ny, mean, nr) || ranges_overlap(y, ny, rstd, nr) ||
        ranges_overlap(mean, nr, rstd, nr) || ranges_overlap(x, nx, mean, nr) || ranges_overlap(x, nx, rstd, nr) || ranges_overlap(gamma, nc, mean, nr) ||
        ranges_overlap(gamma, nc, rstd, nr) || ranges_overlap(beta, nc, mean, nr) || ranges_overlap(beta, nc, rstd, nr))
        return RSDGC_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream_);
    if (dtype == RSDGC_BF16)
        forward_typed<bf16>({static_cast<const bf16 *>(x), gamma, beta, static_cast<bf16 *>(y), mean, rstd, rows, ldx, ldy, static_cast<int32_t>(cols), static_cast<float>(eps)}, s);
    else
        forward_typed<float>({static_cast<const float *>(x), gamma, beta, static_cast<float *>(y), mean, rstd, rows, ldx, ldy, static_cast<int32_t>(cols), static_cast<float>(eps)}, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? RSDGC_OK : remember_hip_error(e, "rsdgc_layer_norm");
}

int rsdgc_layer_norm_backward(int32_t dtype, int64_t rows, int64_t cols, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                              const float *gamma, const float *mean, const float *rstd, void *dx, int64_t lddx, float *dgamma,
                              float *dbeta, int accumulate, void *workspace, void *stream_) {
    if (!sizes_ok(dtype, rows, cols) || lddy < cols || ldx < cols || lddx < cols) return RSDGC_EINVAL;
    const size_t size = type_size(dtype);
    if (!aligned_to(gamma, 4) || !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4)) return RSDGC_EINVAL;
    const bool sums = dgamma || dbeta;
    if (sums && (!workspace || !aligned_to(workspace, 256))) return RSDGC_EINVAL;
    const size_t nc = static_cast<size_t>(cols) * 4, nr = static_cast<size_t>(rows) * 4, nw = sums ? rsdgc_layer_norm_workspace_bytes(rows, cols) : 0;
    if (ranges_overlap(dgamma, nc, dbeta, nc) || ranges_overlap(dgamma, nc, gamma, nc) || ranges_overlap(dbeta, nc, gamma, nc)) return RSDGC_EINVAL;
    if (rows > 0) {
        if (!dy || !x || !dx || !mean || !rstd || !aligned_to(dy, size) || !aligned_to(x, size) || !aligned_to(dx, size) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return RSDGC_EINVAL;
        if (!same_or_apart(dy, lddy, dx, lddx, rows, cols, size) || !same_or_apart(x, ldx, dx, lddx, rows, cols, size)) return RSDGC_EINVAL;
        // what is written may touch nothing else that the call reads or writes
        const size_t n_dx = extent_bytes(rows, cols, lddx, size), n_x = extent_bytes(rows, cols, ldx, size), n_dy = extent_bytes(rows, cols, lddy, size);
        const struct { const void *p; size_t n; } written[] = {{dx, n_dx}, {dgamma, nc}, {dbeta, nc}, {workspace, nw}};
        const struct { const void *p; size_t n; } other[] = {{gamma, nc}, {mean, nr}, {rstd, nr}};
        for (int i = 0; i < 4; ++i) {
            for (const auto &o : other)
                if (ranges_overlap(written[i].p, written[i].n, o.p, o.n)) return RSDGC_EINVAL;
            for (int j = i + 1; j < 4; ++j)
                if (ranges_overlap(written[i].p, written[i].n, written[j].p, written[j].n)) return RSDGC_EINVAL;
            if (i && (ranges_overlap(written[i].p, written[i].n, x, n_x) || ranges_overlap(written[i].p, written[i].n, dy, n_dy))) return RSDGC_EINVAL;
        }
    }
    hipStream_t s = static_cast<hipStream_t>(stream_);
    const int blocks = n_lines(rows, cols);
    float *lines = sums ? static_cast<float *>(workspace) : nullptr;
    if (rows > 0) {
        if (dtype == RSDGC_BF16)
            backward_typed<bf16>({static_cast<const bf16 *>(dy), static_cast<const bf16 *>(x), gamma, mean, rstd, static_cast<bf16 *>(dx), lines, rows, lddy, ldx, lddx,
                                  static_cast<int32_t>(cols)}, blocks, s);
        else
            backward_typed<float>({static_cast<const float *>(dy), static_cast<const float *>(x), gamma, mean, rstd, static_cast<float *>(dx), lines, rows, lddy, ldx, lddx,
                                   static_cast<int32_t>(cols)}, blocks, s);
    }
    if (sums)
        hipLaunchKernelGGL(k_norm_lines, dim3(static_cast<unsigned>((2 * cols + 63) / 64)), dim3(64 * kLineWaves), 0, s, lines, blocks, static_cast<int32_t>(cols), dgamma, dbeta, accumulate);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? RSDGC_OK : remember_hip_error(e, "rsdgc_layer_norm_backward");
}

}  // extern "C"
