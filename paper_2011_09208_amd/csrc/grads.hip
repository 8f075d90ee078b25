// The norm over all gradients of a training step, and clipping by it: in place, or into the SGD update of the weights.  The fused
// backward call (ws_split_fc_bwd_sgd) cannot clip, because the norm is known only when the last gradient is.
//   sumsq = sum over all tensors of g^2;  norm = sqrt(sum of the parts' sumsq);  k = min(1, max_norm / norm)
//   g <- k g,  or  p <- p - lr * k * g
// Bound by HBM: the gradients are read once for the norm; then they are read and written, or read with the weights, which are
// written.  Tables of tensors travel in the kernel arguments, GradTable::MOST or UpdateTable::MOST to a launch.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/whalesplit.h"
#include "gemm_core.h"

namespace ws {

constexpr int GRAD_GROUPS = 2048;            // workgroups of a launch at most, each with one partial sum
constexpr int CLIP_GROUPS = 8192;            // and where nothing is summed (update of 204.8 M bf16 weights with their norm: 317 us with 2048, 305)
constexpr int GRAD_THREADS = 256;
constexpr int GRAD_PIECES = 4;               // of eight elements that a thread has on their way at a time
constexpr int GRAD_CHUNK = 8 * GRAD_PIECES * GRAD_THREADS;     // elements that a workgroup takes at a time

// A tensor with a pitch has its rows cut into chunks, or several rows to a chunk; one without is a single row.
struct GradTensor {
    char* data;
    int64_t ld, cols;                        // elements
    int32_t rows;
    uint32_t end2;                           // chunks of the table up to this tensor's end << 1, + 1: fp32
};
struct ParamTensor {
    char* data;
    int64_t ld2;                             // elements << 1, + 1: fp32
};
// Both hold what fits 4 KiB of kernel arguments.
struct GradTable {
    static constexpr int MOST = 120;
    static constexpr bool PARAMS = false;
    GradTensor t[MOST];
    int32_t n, chunks;
};
struct UpdateTable {
    static constexpr int MOST = 80;
    static constexpr bool PARAMS = true;
    GradTensor t[MOST];
    ParamTensor p[MOST];
    int32_t n, chunks;
};
static_assert(sizeof(GradTable) + 64 <= 4096 && sizeof(UpdateTable) + 64 <= 4096, "kernel arguments");

typedef float f32x8[8];

// Elements [at, at + 8) of a row of `len`, those outside [0, len) as zeros; 16 bytes at a time where the address allows.
template <typename T>
__device__ __forceinline__ void read8(const T* row, int at, int len, bool wide, f32x8& f) {
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
__device__ __forceinline__ void write8(T* row, int at, int len, bool wide, const f32x8& f) {
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

// Calls f(tensor number, first row, rows, from, to) for every chunk of elements [from, to) of rows that this workgroup owns, chunks blockIdx.x,
// + gridDim.x, .. counted from the first tensor on, or from the last one backwards.  The lanes look at all tensors at once for the one that holds a chunk: going
// through them took 5 of the 21 us of 25 M gradients in 96 tensors.
template <bool BACKWARDS, class Table, class F>
__device__ __forceinline__ void for_each_chunk(const Table& table, F f) {
    static_assert(Table::MOST <= 128, "");
    const int lane = threadIdx.x & 63;
    const int32_t end_a = lane < table.n ? (int32_t)(table.t[lane].end2 >> 1) : INT_MAX;
    const int32_t end_b = lane + 64 < table.n ? (int32_t)(table.t[lane + 64 < Table::MOST ? lane + 64 : 0].end2 >> 1) : INT_MAX;
    for (int32_t i = blockIdx.x; i < table.chunks; i += gridDim.x) {
        const int32_t at = BACKWARDS ? table.chunks - 1 - i : i;
        const int t = __builtin_amdgcn_readfirstlane((int)(__popcll(__ballot(end_a <= at)) + __popcll(__ballot(end_b <= at))));
        const GradTensor& d = table.t[t];
        const int32_t c = at - (t > 0 ? (int32_t)(table.t[t - 1].end2 >> 1) : 0);
        if (d.rows == 1) {                                   // chunks at 16-byte boundaries
            const int64_t from = (int64_t)c * GRAD_CHUNK - ((reinterpret_cast<uintptr_t>(d.data) & 15) >> (d.end2 & 1 ? 2 : 1));
            f(t, 0, 1, from > 0 ? from : 0, from + GRAD_CHUNK < d.cols ? from + GRAD_CHUNK : d.cols);
        } else if (d.cols > GRAD_CHUNK / 2) {
            const int32_t per_row = (int32_t)((d.cols + GRAD_CHUNK - 1) / GRAD_CHUNK), row = c / per_row;
            const int64_t from = (int64_t)(c - row * per_row) * GRAD_CHUNK;
            f(t, row, 1, from, from + GRAD_CHUNK < d.cols ? from + GRAD_CHUNK : d.cols);
        } else {
            const int32_t per = GRAD_CHUNK / (int32_t)d.cols, row = c * per;
            f(t, row, d.rows - row < per ? d.rows - row : per, (int64_t)0, d.cols);
        }
    }
}

// Calls f(row, at) for pieces [at, at + 8) that cover elements [0, len) of each row; they start at 16-byte boundaries, so the first and the last of a row may
// hang over its ends.
template <typename T, class F>
__device__ __forceinline__ void for_each_piece(const T* data, int64_t ld, int rows, int len, F f) {
    const int per_row = ((len + 7) >> 3) + 1;
    for (int u = threadIdx.x; u < rows * per_row; u += GRAD_THREADS) {
        const int r = rows == 1 ? 0 : u / per_row;
        f(r, 8 * (u - r * per_row) - misaligned(data + r * ld));
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
__device__ __forceinline__ double add_squares(double sum, const f32x8& v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)v[e], (double)v[e], sum);
    return sum;
}

// A whole chunk at a 16-byte boundary has its loads side by side: 8.4 M bf16 gradients in 48 tensors took 18.6 us with a branch around each.
__global__ __launch_bounds__(GRAD_THREADS) void grad_sumsq(GradTable table, double* __restrict__ parts) {
    __shared__ double part[GRAD_THREADS / 64];
    double sum = 0.0;
    for_each_chunk<false>(table, [&](int t, int row0, int rows, int64_t from, int64_t to) {
        const int64_t ld = table.t[t].ld;
        const bool wide = table.t[t].end2 & 1;
        const char* first = table.t[t].data + (row0 * ld + from) * (wide ? 4 : 2);
        const int len = (int)(to - from);
        auto add = [&](auto type) {
            typedef decltype(type) T;
            const T* g = reinterpret_cast<const T*>(first);
            if (len == GRAD_CHUNK && misaligned(g) == 0) {                               // then there is one row
                const T* mine = g + 8 * threadIdx.x;
                f32x8 v[GRAD_PIECES];
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) read8(mine, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, v[i]);
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) sum = add_squares(sum, v[i]);
                return;
            }
            for_each_piece(g, ld, rows, len, [&](int row, int at) {
                f32x8 v;
                read8(g + row * ld, at, len, true, v);
                sum = add_squares(sum, v);
            });
        };
        if (wide) add(float{});
        else add(uint16_t{});
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

// k of the clipping rule, 0 for a norm that is not finite; the first workgroup also reports the norm.  k g is at most max_norm, an ordinary number, where k
// itself may be far below fp32's range: such a factor is applied in 64 bits.
struct ClipFactor {
    double k;
    float k32;
    bool tiny;
    __device__ __forceinline__ ClipFactor(const double* sumsq, int S, float max_norm, float* norm) {
        double total = 0.0;
        for (int s = 0; s < S; ++s) total += sumsq[s];
        const double n = sqrt(total);
        if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
        k = !(n <= 1.7976931348623157e308) ? 0.0 : n > (double)max_norm ? (double)max_norm / n : 1.0;
        k32 = (float)k;
        tiny = k < 1.1754943508222875e-38;                   // 2^-126
    }
    // v <- k v; a factor of 0 leaves no NaN behind
    __device__ __forceinline__ void apply(f32x8& v) const {
        if (tiny) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k == 0.0 ? 0.0f : (float)(k * (double)v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= k32;
        }
    }
};

// The tensors are taken backwards: what the sum of squares has read last may still be in the Infinity Cache.  Clipping 204.8 M bf16 gradients takes 153 us (5.4 TB/s
// read and written), 33.6 M fp32 42 (6.4), 37.8 M bf16 in 95 tensors 25 (6.0).
__global__ __launch_bounds__(GRAD_THREADS) void grad_clip(GradTable table, const double* __restrict__ sumsq, int S, float max_norm,
                                                          float* __restrict__ norm) {
    const ClipFactor factor(sumsq, S, max_norm, norm);
    if (factor.k32 == 1.0f) return;
    for_each_chunk<true>(table, [&](int t, int row0, int rows, int64_t from, int64_t to) {
        const int64_t ld = table.t[t].ld;
        const bool wide = table.t[t].end2 & 1;
        char* first = table.t[t].data + (row0 * ld + from) * (wide ? 4 : 2);
        const int len = (int)(to - from);
        auto scale = [&](auto type) {
            typedef decltype(type) T;
            T* g = reinterpret_cast<T*>(first);
            if (len == GRAD_CHUNK && misaligned(g) == 0) {
                T* mine = g + 8 * threadIdx.x;
                f32x8 v[GRAD_PIECES];
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) read8(mine, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, v[i]);
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) {
                    factor.apply(v[i]);
                    write8(mine, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, v[i]);
                }
                return;
            }
            for_each_piece(g, ld, rows, len, [&](int row, int at) {
                f32x8 v;
                read8(g + row * ld, at, len, true, v);
                factor.apply(v);
                write8(g + row * ld, at, len, true, v);
            });
        };
        if (wide) scale(float{});
        else scale(uint16_t{});
    });
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_sgd(UpdateTable table, const double* __restrict__ sumsq, int S, float max_norm, float lr,
                                                              float* __restrict__ norm) {
    const ClipFactor factor(sumsq, S, max_norm, norm);
    if (factor.k == 0.0) return;                             // a step without a finite norm changes nothing
    for_each_chunk<true>(table, [&](int t, int row0, int rows, int64_t from, int64_t to) {
        const int64_t ldg = table.t[t].ld, ldp = table.p[t].ld2 >> 1;
        const bool wide_g = table.t[t].end2 & 1, wide_p = table.p[t].ld2 & 1;
        const char* g0 = table.t[t].data + (row0 * ldg + from) * (wide_g ? 4 : 2);
        char* p0 = table.p[t].data + (row0 * ldp + from) * (wide_p ? 4 : 2);
        const int len = (int)(to - from);
        auto update = [&](auto g_type, auto p_type) {
            typedef decltype(g_type) G;
            typedef decltype(p_type) P;
            const G* g = reinterpret_cast<const G*>(g0);
            P* p = reinterpret_cast<P*>(p0);
            auto updated = [&](f32x8& w, f32x8& v) {
                factor.apply(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = fmaf(-lr, v[e], w[e]);
            };
            if (len == GRAD_CHUNK && ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(p)) & 15) == 0) {       // then there is one row
                const G* mine = g + 8 * threadIdx.x;
                P* own = p + 8 * threadIdx.x;
                f32x8 v[GRAD_PIECES], w[GRAD_PIECES];
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) {
                    read8(mine, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, v[i]);
                    read8(own, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, w[i]);
                }
#pragma unroll
                for (int i = 0; i < GRAD_PIECES; ++i) {
                    updated(w[i], v[i]);
                    write8(own, 8 * GRAD_THREADS * i, GRAD_CHUNK, true, w[i]);
                }
                return;
            }
            for_each_piece(g, ldg, rows, len, [&](int row, int at) {
                P* own = p + (int64_t)row * ldp;
                const bool wide = misaligned(own + at) == 0;
                f32x8 v, w;
                read8(g + (int64_t)row * ldg, at, len, true, v);
                read8(own, at, len, wide, w);
                updated(w, v);
                write8(own, at, len, wide, w);
            });
        };
        if (wide_g) {
            if (wide_p) update(float{}, float{});
            else update(float{}, uint16_t{});
        } else {
            if (wide_p) update(uint16_t{}, float{});
            else update(uint16_t{}, uint16_t{});
        }
    });
}

struct TensorList {
    const void* const* data;
    const int64_t *rows, *cols, *ld;
    const int32_t* bytes;
};

// Chunks of a tensor as the kernels count them, for_each_chunk.
static int64_t chunks_of(const void* data, int64_t rows, int64_t cols, int32_t bytes) {
    if (rows == 1) return (cols + (int64_t)((reinterpret_cast<uintptr_t>(data) & 15) >> (bytes == 4 ? 2 : 1)) + GRAD_CHUNK - 1) / GRAD_CHUNK;
    if (cols > GRAD_CHUNK / 2) return rows * ((cols + GRAD_CHUNK - 1) / GRAD_CHUNK);
    return (rows + GRAD_CHUNK / cols - 1) / (GRAD_CHUNK / cols);
}

// Checks tensors [0, n); empty ones may have no data.
static int check_tensors(const TensorList& l, int32_t n) {
    if (n == 0) return WS_OK;
    if (!l.data || !l.rows || !l.cols || !l.ld || !l.bytes) return WS_ERR_NULL;
    for (int i = 0; i < n; ++i) {
        if (l.rows[i] < 0 || l.cols[i] < 0 || (l.bytes[i] != 2 && l.bytes[i] != 4)) return WS_ERR_SHAPE;
        if (l.rows[i] == 0 || l.cols[i] == 0) continue;
        if (!l.data[i]) return WS_ERR_NULL;
        if (l.rows[i] > INT32_MAX || (l.rows[i] > 1 && l.ld[i] < l.cols[i])) return WS_ERR_SHAPE;
        // chunks are counted in 30 bits
        if (l.cols[i] > (int64_t)1 << 42 || (l.rows[i] > 1 && l.cols[i] > ((int64_t)1 << 42) / l.rows[i])) return WS_ERR_RANGE;
        if (l.rows[i] > 1 && chunks_of(l.data[i], l.rows[i], l.cols[i], l.bytes[i]) > INT32_MAX / 2) return WS_ERR_RANGE;
        if (reinterpret_cast<uintptr_t>(l.data[i]) & (uintptr_t)(l.bytes[i] - 1)) return WS_ERR_ALIGN;
    }
    return WS_OK;
}

// Calls launch(table, groups) for as many tensors that hold something as a table takes, from the first on or from the last; returns a status.
// `p` are the parameters of an UpdateTable.
template <class Table, class F>
static int for_each_table(const TensorList& g, const TensorList* p, int32_t n, bool backwards, F launch) {
    Table table;
    table.n = 0;
    int64_t chunks = 0;
    auto flush = [&]() {
        if (table.n == 0) return (int)WS_OK;
        table.chunks = (int32_t)chunks;
        const int most = backwards ? CLIP_GROUPS : GRAD_GROUPS;
        launch(table, (unsigned)(chunks < most ? chunks : most));
        table.n = 0;
        chunks = 0;
        return hipGetLastError() == hipSuccess ? (int)WS_OK : (int)WS_ERR_HIP;
    };
    for (int j = 0; j < n; ++j) {
        const int i = backwards ? n - 1 - j : j;
        int64_t rows = g.rows[i], cols = g.cols[i];
        if (rows == 0 || cols == 0) continue;
        if (rows > 1 && g.ld[i] == cols && (!p || p->ld[i] == cols)) {             // one long row
            cols *= rows;
            rows = 1;
        }
        const int64_t mine = chunks_of(g.data[i], rows, cols, g.bytes[i]);
        if (chunks + mine > INT32_MAX / 2 || table.n == Table::MOST) {
            const int st = flush();
            if (st != WS_OK) return st;
        }
        GradTensor& t = table.t[table.n];
        t.data = static_cast<char*>(const_cast<void*>(g.data[i]));
        t.ld = g.ld[i];
        t.cols = cols;
        t.rows = (int32_t)rows;
        t.end2 = (uint32_t)(chunks + mine) << 1 | (g.bytes[i] == 4);
        if constexpr (Table::PARAMS) {
            table.p[table.n].data = static_cast<char*>(const_cast<void*>(p->data[i]));
            table.p[table.n].ld2 = p->ld[i] << 1 | (p->bytes[i] == 4);
        }
        ++table.n;
        chunks += mine;
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
    return n < 0 ? 0 : ((size_t)(n + GradTable::MOST - 1) / GradTable::MOST + 1) * GRAD_GROUPS * sizeof(double);
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
    st = for_each_table<GradTable>(g, nullptr, n, false, [&](const GradTable& table, unsigned groups) {
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
    st = for_each_table<GradTable>(g, nullptr, n, true, [&](const GradTable& table, unsigned groups) {
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
    st = for_each_table<UpdateTable>(g, &p, n, true, [&](const UpdateTable& table, unsigned groups) {
        hipLaunchKernelGGL(grad_clip_sgd, dim3(groups), dim3(GRAD_THREADS), 0, s, table, sumsq, S, max_norm, lr, told ? nullptr : norm);
        told = true;
    });
    if (st != WS_OK || told || !norm) return st;
    hipLaunchKernelGGL(grad_clip_sgd, dim3(1), dim3(GRAD_THREADS), 0, s, UpdateTable{}, sumsq, S, max_norm, lr, norm);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

}  // extern "C"
