// The norm over all gradients of a training step, and clipping by it: in place, or into the SGD update of the weights.  The fused
// backward call (ws_split_fc_bwd_sgd) cannot clip, because the norm is known only when the last gradient is.
//   sumsq = sum over all tensors of g^2;  norm = sqrt(sum of the parts' sumsq);  k = min(1, max_norm / norm)
//   g <- k g,  or  p <- p - lr * k * g
// Bound by HBM: the gradients are read once for the norm; then they are read and written, or read with the weights, which are
// written.  Tables of tensors travel in the kernel arguments, GRAD_TENSORS to a launch.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/whalesplit.h"
#include "gemm_core.h"

namespace ws {

constexpr int GRAD_TENSORS = 48;
constexpr int GRAD_GROUPS = 1024;            // workgroups of a launch at most, each with one partial sum
constexpr int GRAD_THREADS = 256;
constexpr int GRAD_CHUNK = 8192;             // elements that a workgroup takes at a time

struct GradTensor {
    char* g;                                 // gradients, bf16 or fp32
    char* p;                                 // parameters, or nullptr
    int64_t ldg, ldp, cols;                  // elements
    int32_t rows, chunks;
    uint16_t g_bytes, p_bytes;
    uint32_t row_chunks;                     // chunks of a row, or 0: `per` rows to a chunk
    int32_t per;
};
struct GradTable {
    GradTensor t[GRAD_TENSORS];
    int32_t n, chunks;
};
static_assert(sizeof(GradTable) + 64 <= 4096, "kernel arguments");

typedef float f32x8[8];

// Elements [at, at + 8) of a row of `len`, those outside [0, len) as zeros; 16 bytes at a time where the address allows.
template <typename T>
__device__ __forceinline__ void read8(const T* row, int64_t at, int64_t len, bool wide, f32x8& f) {
    if (wide && at >= 0 && at + 8 <= len) {
        if constexpr (sizeof(T) == 2) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(row + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[2 * e] = __uint_as_float(v[e] << 16);
                f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            }
        } else {
            const f32x4 a = reinterpret_cast<const f32x4*>(row + at)[0], b = reinterpret_cast<const f32x4*>(row + at)[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = a[e];
                f[4 + e] = b[e];
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = 0.0f;
        if (at + e >= 0 && at + e < len) {
            if constexpr (sizeof(T) == 2) f[e] = __uint_as_float((uint32_t)row[at + e] << 16);
            else f[e] = row[at + e];
        }
    }
}
template <typename T>
__device__ __forceinline__ void write8(T* row, int64_t at, int64_t len, bool wide, const f32x8& f) {
    if (wide && at >= 0 && at + 8 <= len) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4*>(row + at) = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
        } else {
            reinterpret_cast<f32x4*>(row + at)[0] = f32x4{f[0], f[1], f[2], f[3]};
            reinterpret_cast<f32x4*>(row + at)[1] = f32x4{f[4], f[5], f[6], f[7]};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e >= 0 && at + e < len) {
            if constexpr (sizeof(T) == 2) row[at + e] = (uint16_t)pack_bf16(f[e], 0.0f);
            else row[at + e] = f[e];
        }
}

// Elements from the last 16-byte boundary at or before a pointer to the pointer.
template <typename T>
__device__ __forceinline__ int misaligned(const T* p) { return (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T); }

// Calls f(row, from, to) for every run of elements [from, to) of a row that this workgroup owns, chunks blockIdx.x, + gridDim.x, ..
template <class F>
__device__ __forceinline__ void for_each_run(const GradTable& table, F f) {
    int t = 0, first = 0;
    for (int64_t chunk = blockIdx.x; chunk < table.chunks; chunk += gridDim.x) {
        while (chunk >= first + table.t[t].chunks) first += table.t[t++].chunks;
        const GradTensor& d = table.t[t];
        const uint32_t c = (uint32_t)(chunk - first);
        if (d.row_chunks > 0) {
            const uint32_t row = c / d.row_chunks;
            const int64_t from = (int64_t)(c - row * d.row_chunks) * GRAD_CHUNK;
            f(d, (int)row, 1, from, from + GRAD_CHUNK < d.cols ? from + GRAD_CHUNK : d.cols);
        } else {
            const int row = (int)c * d.per;
            f(d, row, d.rows - row < d.per ? d.rows - row : d.per, (int64_t)0, d.cols);
        }
    }
}

// Eight elements of the run at a time; pieces start at 16-byte boundaries of G.  Calls f(row, at, wide): elements [at, at + 8) of the row,
// of which those outside [0, d.cols) and outside the run are not there.
template <typename T, class F>
__device__ __forceinline__ void for_each_piece(const GradTensor& d, int row0, int rows, int64_t from, int64_t to, F f) {
    const int per_row = (int)((to - from + 7) >> 3) + 1;
    for (int u = threadIdx.x; u < rows * per_row; u += GRAD_THREADS) {
        const int r = rows == 1 ? 0 : u / per_row;
        const T* g = reinterpret_cast<const T*>(d.g) + (int64_t)(row0 + r) * d.ldg + from;
        f(row0 + r, 8 * (int64_t)(u - r * per_row) - misaligned(g));
    }
}

__device__ __forceinline__ double block_sum(double v, double* part) {
    for (int w = 32; w > 0; w >>= 1) v += __shfl_xor(v, w, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) v += part[w];
    return v;
}

// Squares are summed in 64 bits: those of finite fp32 gradients neither overflow nor vanish, and a sum over 10^9 of them is right to fp32.
__global__ __launch_bounds__(GRAD_THREADS) void grad_sumsq(GradTable table, double* __restrict__ parts) {
    __shared__ double part[GRAD_THREADS / 64];
    double sum = 0.0;
    for_each_run(table, [&](const GradTensor& d, int row0, int rows, int64_t from, int64_t to) {
        auto add = [&](auto type) {
            typedef decltype(type) T;
            for_each_piece<T>(d, row0, rows, from, to, [&](int row, int64_t at) {
                const T* g = reinterpret_cast<const T*>(d.g) + (int64_t)row * d.ldg + from;
                f32x8 v;
                read8(g, at, to - from, true, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fma((double)v[e], (double)v[e], sum);
            });
        };
        if (d.g_bytes == 2) add(uint16_t{});
        else add(float{});
    });
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_sumsq_total(const double* __restrict__ parts, int n, double* __restrict__ sumsq) {
    __shared__ double part[16];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 1024) sum += parts[i];
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) *sumsq = sum;
}

// k of the clipping rule, 0 for a norm that is not finite; the first workgroup also reports the norm.
__device__ __forceinline__ float clip_factor(const double* sumsq, int S, float max_norm, float* norm) {
    double total = 0.0;
    for (int s = 0; s < S; ++s) total += sumsq[s];
    const double n = sqrt(total);
    if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    if (!(n <= 1.7976931348623157e308)) return 0.0f;
    return n > (double)max_norm ? (float)((double)max_norm / n) : 1.0f;
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_clip(GradTable table, const double* __restrict__ sumsq, int S, float max_norm,
                                                          float* __restrict__ norm) {
    const float k = clip_factor(sumsq, S, max_norm, norm);
    if (k == 1.0f) return;
    for_each_run(table, [&](const GradTensor& d, int row0, int rows, int64_t from, int64_t to) {
        auto scale = [&](auto type) {
            typedef decltype(type) T;
            for_each_piece<T>(d, row0, rows, from, to, [&](int row, int64_t at) {
                T* g = reinterpret_cast<T*>(d.g) + (int64_t)row * d.ldg + from;
                f32x8 v;
                read8(g, at, to - from, true, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k == 0.0f ? 0.0f : k * v[e];      // a factor of 0 leaves no NaN behind
                write8(g, at, to - from, true, v);
            });
        };
        if (d.g_bytes == 2) scale(uint16_t{});
        else scale(float{});
    });
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_sgd(GradTable table, const double* __restrict__ sumsq, int S, float max_norm, float lr,
                                                              float* __restrict__ norm) {
    const float k = clip_factor(sumsq, S, max_norm, norm);
    if (k == 0.0f) return;                                   // a step without a finite norm changes nothing
    for_each_run(table, [&](const GradTensor& d, int row0, int rows, int64_t from, int64_t to) {
        auto update = [&](auto g_type, auto p_type) {
            typedef decltype(g_type) G;
            typedef decltype(p_type) P;
            for_each_piece<G>(d, row0, rows, from, to, [&](int row, int64_t at) {
                const G* g = reinterpret_cast<const G*>(d.g) + (int64_t)row * d.ldg + from;
                P* p = reinterpret_cast<P*>(d.p) + (int64_t)row * d.ldp + from;
                const bool wide = misaligned(p + at) == 0;
                f32x8 v, w;
                read8(g, at, to - from, true, v);
                read8(p, at, to - from, wide, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = fmaf(-lr, k * v[e], w[e]);
                write8(p, at, to - from, wide, w);
            });
        };
        if (d.g_bytes == 2 && d.p_bytes == 2) update(uint16_t{}, uint16_t{});
        else if (d.g_bytes == 2) update(uint16_t{}, float{});
        else if (d.p_bytes == 2) update(float{}, uint16_t{});
        else update(float{}, float{});
    });
}

struct TensorList {
    const void* const* data;
    const int64_t *rows, *cols, *ld;
    const int32_t* bytes;
};

// Checks tensors [0, n); empty ones may have no data.
static int check_tensors(const TensorList& l, int32_t n) {
    if (n == 0) return WS_OK;
    if (!l.data || !l.rows || !l.cols || !l.ld || !l.bytes) return WS_ERR_NULL;
    for (int i = 0; i < n; ++i) {
        if (l.rows[i] < 0 || l.cols[i] < 0 || (l.bytes[i] != 2 && l.bytes[i] != 4)) return WS_ERR_SHAPE;
        if (l.rows[i] == 0 || l.cols[i] == 0) continue;
        if (!l.data[i]) return WS_ERR_NULL;
        if (l.rows[i] > INT32_MAX || (l.rows[i] > 1 && l.ld[i] < l.cols[i])) return WS_ERR_SHAPE;
        if (l.cols[i] > ((int64_t)1 << 42) / l.rows[i]) return WS_ERR_RANGE;       // chunks are counted in 31 bits
        if (reinterpret_cast<uintptr_t>(l.data[i]) % (uintptr_t)l.bytes[i]) return WS_ERR_ALIGN;
    }
    return WS_OK;
}

// Calls launch(table, groups) for every GRAD_TENSORS tensors that hold something; returns a status.
template <class F>
static int for_each_table(const TensorList& g, const TensorList* p, int32_t n, F launch) {
    GradTable table = {};
    int64_t chunks = 0;
    auto flush = [&]() {
        if (chunks == 0) return (int)WS_OK;
        if (chunks > INT32_MAX) return (int)WS_ERR_RANGE;
        table.chunks = (int32_t)chunks;
        launch(table, (unsigned)(chunks < GRAD_GROUPS ? chunks : GRAD_GROUPS));
        table = GradTable{};
        chunks = 0;
        return hipGetLastError() == hipSuccess ? (int)WS_OK : (int)WS_ERR_HIP;
    };
    for (int i = 0; i < n; ++i) {
        if (g.rows[i] == 0 || g.cols[i] == 0) continue;
        GradTensor& t = table.t[table.n++];
        t.g = static_cast<char*>(const_cast<void*>(g.data[i]));
        t.ldg = g.ld[i];
        t.g_bytes = (uint16_t)g.bytes[i];
        t.p = p ? static_cast<char*>(const_cast<void*>(p->data[i])) : nullptr;
        t.ldp = p ? p->ld[i] : 0;
        t.p_bytes = p ? (uint16_t)p->bytes[i] : 0;
        int64_t rows = g.rows[i], cols = g.cols[i];
        if (rows > 1 && t.ldg == cols && (!p || t.ldp == cols)) {                  // one long row
            cols *= rows;
            rows = 1;
        }
        t.rows = (int32_t)rows;
        t.cols = cols;
        const int64_t row_chunks = (cols + GRAD_CHUNK - 1) / GRAD_CHUNK;
        const int64_t fit = GRAD_CHUNK / cols;
        t.row_chunks = rows == 1 || fit < 2 ? (uint32_t)row_chunks : 0;
        t.per = t.row_chunks ? 1 : (int32_t)fit;
        const int64_t mine = t.row_chunks ? rows * row_chunks : (rows + fit - 1) / fit;
        if (mine > INT32_MAX) return WS_ERR_RANGE;
        t.chunks = (int32_t)mine;
        chunks += mine;
        if (table.n == GRAD_TENSORS) {
            const int st = flush();
            if (st != WS_OK) return st;
        }
    }
    return flush();
}

static int check_clip(const double* sumsq, int32_t S, float max_norm, const float* norm) {
    if (!sumsq) return WS_ERR_NULL;
    if (S < 1 || S > WS_GRAD_MAX_PARTS || !(max_norm > 0.0f)) return WS_ERR_RANGE;
    if (reinterpret_cast<uintptr_t>(sumsq) % 8 || reinterpret_cast<uintptr_t>(norm) % 4) return WS_ERR_ALIGN;
    return WS_OK;
}

}  // namespace ws

using namespace ws;

extern "C" {

size_t ws_grad_workspace_bytes(int32_t n) {
    return n < 0 ? 0 : ((size_t)(n + GRAD_TENSORS - 1) / GRAD_TENSORS + 1) * GRAD_GROUPS * sizeof(double);
}

int ws_grad_sumsq(const void* const* grads, const int64_t* rows, const int64_t* cols, const int64_t* lds, const int32_t* elem_bytes, int32_t n,
                  double* sumsq, void* workspace, size_t workspace_bytes, void* stream) {
    if (!sumsq) return WS_ERR_NULL;
    if (n < 0) return WS_ERR_RANGE;
    const TensorList g = {grads, rows, cols, lds, elem_bytes};
    int st = check_tensors(g, n);
    if (st != WS_OK) return st;
    if (reinterpret_cast<uintptr_t>(sumsq) % 8) return WS_ERR_ALIGN;
    if (!workspace || workspace_bytes < ws_grad_workspace_bytes(n)) return WS_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return WS_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double* parts = static_cast<double*>(workspace);
    int used = 0;
    st = for_each_table(g, nullptr, n, [&](const GradTable& table, unsigned groups) {
        hipLaunchKernelGGL(grad_sumsq, dim3(groups), dim3(GRAD_THREADS), 0, s, table, parts + used);
        used += (int)groups;
    });
    if (st != WS_OK) return st;
    hipLaunchKernelGGL(grad_sumsq_total, dim3(1), dim3(1024), 0, s, parts, used, sumsq);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

int ws_grad_clip(void* const* grads, const int64_t* rows, const int64_t* cols, const int64_t* lds, const int32_t* elem_bytes, int32_t n,
                 const double* sumsq, int32_t S, float max_norm, float* norm, void* stream) {
    if (n < 0) return WS_ERR_RANGE;
    const TensorList g = {const_cast<const void* const*>(grads), rows, cols, lds, elem_bytes};
    int st = check_tensors(g, n);
    if (st == WS_OK) st = check_clip(sumsq, S, max_norm, norm);
    if (st != WS_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    bool told = false;
    st = for_each_table(g, nullptr, n, [&](const GradTable& table, unsigned groups) {
        hipLaunchKernelGGL(grad_clip, dim3(groups), dim3(GRAD_THREADS), 0, s, table, sumsq, S, max_norm, told ? nullptr : norm);
        told = true;
    });
    if (st != WS_OK || told || !norm) return st;
    hipLaunchKernelGGL(grad_clip, dim3(1), dim3(GRAD_THREADS), 0, s, GradTable{}, sumsq, S, max_norm, norm);     // nothing but the norm
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

int ws_grad_clip_sgd(void* const* params, const int64_t* ld_params, const int32_t* param_bytes, const void* const* grads, const int64_t* rows,
                     const int64_t* cols, const int64_t* lds, const int32_t* elem_bytes, int32_t n, const double* sumsq, int32_t S, float max_norm,
                     float lr, float* norm, void* stream) {
    if (n < 0) return WS_ERR_RANGE;
    const TensorList g = {grads, rows, cols, lds, elem_bytes};
    const TensorList p = {const_cast<const void* const*>(params), rows, cols, ld_params, param_bytes};
    int st = check_tensors(g, n);
    if (st == WS_OK) st = check_tensors(p, n);
    if (st == WS_OK) st = check_clip(sumsq, S, max_norm, norm);
    if (st != WS_OK) return st;
    if (!isfinite(lr)) return WS_ERR_RANGE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    bool told = false;
    st = for_each_table(g, &p, n, [&](const GradTable& table, unsigned groups) {
        hipLaunchKernelGGL(grad_clip_sgd, dim3(groups), dim3(GRAD_THREADS), 0, s, table, sumsq, S, max_norm, lr, told ? nullptr : norm);
        told = true;
    });
    if (st != WS_OK || told || !norm) return st;
    hipLaunchKernelGGL(grad_clip_sgd, dim3(1), dim3(GRAD_THREADS), 0, s, GradTable{}, sumsq, S, max_norm, lr, norm);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

}  // extern "C"
