// Root-mean-square norm around the split layer: what turns the residual stream of a language model into the features X,
// and the way back for the gradient that the shards leave (ws_split_fc_bwd, ws_bridge_reduce_partition).
//   h = residual + x (rounded to the stream's type),  y = h * rstd * gamma,  rstd = 1 / sqrt(mean(h^2) + eps)
//   dh = dres + rstd * (gamma * dY - xhat * mean(gamma * dY * xhat)),  dgamma = sum over the rows of dY * xhat,  xhat = h * rstd
// Bound by HBM: every value is read and written once, a row is held in registers between its sum and its result.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/whalesplit.h"
#include "mx.h"

namespace ws {

constexpr int NORM_MAX_D = WS_RMS_NORM_MAX_D;

struct NormArgs {
    const uint16_t* x; int64_t ldx;
    const void* res; int64_t ldr;        // stream type, or nullptr
    const float* gamma;
    float eps;
    int B, D;
    void* h; int64_t ldh;                // stream type, or nullptr
    void* y; int64_t ldy;                // bf16 or e4m3
    uint8_t* scales; int64_t lds;
    float* rstd;                         // or nullptr
};

typedef float f32x8[8];

__device__ __forceinline__ void unpack8(u32x4 v, f32x8& f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(v[e] << 16);
        f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ u32x4 pack8(const f32x8& f) {
    return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}
__device__ __forceinline__ void load8(const float* p, f32x8& f) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = a[e];
        f[4 + e] = b[e];
    }
}
__device__ __forceinline__ void store8(float* p, const f32x8& f) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{f[0], f[1], f[2], f[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{f[4], f[5], f[6], f[7]};
}
// Eight values of a stream row, bf16 or fp32.
template <bool FP32>
__device__ __forceinline__ void load_stream(const void* base, int64_t at, f32x8& f) {
    if constexpr (FP32) load8(static_cast<const float*>(base) + at, f);
    else unpack8(*reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at), f);
}
template <bool FP32>
__device__ __forceinline__ void store_stream(void* base, int64_t at, const f32x8& f) {
    if constexpr (FP32) store8(static_cast<float*>(base) + at, f);
    else *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + at) = pack8(f);
}

// Sum over groups of T neighbouring lanes, the same in all of them and in the same order whatever the lane.
template <int T>
__device__ __forceinline__ float lane_sum(float v) {
    v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xF, 0xF, true));     // lane ^ 1
    v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xF, 0xF, true));     // lane ^ 2
    v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x141, 0xF, 0xF, true));    // the other quad of eight
    if (T >= 16) v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x140, 0xF, 0xF, true));    // the other half of sixteen
    if (T >= 32) v += __shfl_xor(v, 16, 64);
    if (T >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

// Sum over the T threads of a row; T > 64: the whole workgroup, which meets at a barrier.  `part` is not read again before the next
// call's barrier if calls alternate between two of them.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* part) {
    v = lane_sum<T>(v);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) v += part[w];
    }
    return v;
}

// T threads take a row, NV pieces of eight features each, in steps of 8 T: D <= 8 T NV.  A wave for a row needs no barrier; short rows share one (the
// rows of a norm over 64 features: 65 536 of them 23.5 us with a wave for each).
template <int T, int NV, bool FP32, bool MX>
__global__ __launch_bounds__(T > 256 ? T : 256) void rms_norm_fwd(NormArgs a) {
    constexpr int ROWS = T > 256 ? 1 : 256 / T;
    __shared__ float part[T > 64 ? T / 64 : 1];
    const int t = threadIdx.x % T;
    const int row = blockIdx.x * ROWS + threadIdx.x / T;
    if (T <= 64 && row >= a.B) return;                     // T > 64: one row to a workgroup, and as many workgroups as rows
    const int n = a.D >> 3;
    const uint16_t* x = a.x + row * a.ldx;
    f32x8 h[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = t + k * T;
        if (c < n) unpack8(*reinterpret_cast<const u32x4*>(x + 8 * c), h[k]);
    }
    if (a.res != nullptr) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t + k * T;
            f32x8 r;
            if (c < n) {
                load_stream<FP32>(a.res, row * a.ldr + 8 * c, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k][e] += r[e];
                if constexpr (!FP32) unpack8(pack8(h[k]), h[k]);      // what the stream stores is what is normalised
            }
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = t + k * T;
        if (c < n) {
            if (a.h != nullptr) store_stream<FP32>(a.h, row * a.ldh + 8 * c, h[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(h[k][e], h[k][e], sum);
        }
    }
    sum = row_sum<T>(sum, part);
    const float rstd = 1.0f / sqrtf(sum / (float)a.D + a.eps);
    if (a.rstd != nullptr && t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = t + k * T;
        if (c >= n) continue;
        f32x8 g;
        load8(a.gamma + 8 * c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] *= h[k][e] * rstd;
        if constexpr (!MX) {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + row * a.ldy + 8 * c) = pack8(g);
        } else {
            // four lanes hold the 32 values of a group; D is a multiple of 64, so they are all there or none
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = __float_as_uint(g[e]) & 0x7fffffffu;
                top = top > m ? top : m;
            }
            const uint32_t byte = group_scale<E4M3_TOP_EXPONENT, E4M3_TOP_FRACTION>(quad_max(top));
            const float inv = inverse_scale(byte);
            u32x2 q;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                int v = __builtin_amdgcn_cvt_pk_fp8_f32(g[4 * e] * inv, g[4 * e + 1] * inv, 0, false);
                v = __builtin_amdgcn_cvt_pk_fp8_f32(g[4 * e + 2] * inv, g[4 * e + 3] * inv, v, true);
                q[e] = (uint32_t)v;
            }
            *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.y) + row * a.ldy + 8 * c) = q;
            if ((c & 3) == 0) a.scales[row * a.lds + (c >> 2)] = (uint8_t)byte;
        }
    }
}

struct NormBackArgs {
    const float* dY; int64_t lddy;
    const void* h; int64_t ldh;
    const void* dres; int64_t ldd;       // or nullptr
    const float* gamma;
    const float* rstd;
    int B, D;
    void* dh; int64_t lddh;
    float* parts;                        // [gridDim.x][D], or nullptr: dgamma is not wanted
};

// A workgroup walks rows blockIdx.x * ROWS + .., gridDim.x * ROWS apart, and keeps its share of dgamma in registers: a thread's
// columns are the same in every row.  Where a wave takes a row, eight waves add theirs up: every share costs a write and a read of D floats
// (1024 x 2048, this kernel alone, with four waves: 11.0 us).  All eight shares meet in LDS at once and the threads share out the columns: 7.4 us, in
// pairs and pairs of pairs 8.4; with the next row's loads ahead 6.3.  The sum of the 128 shares, in 64 workgroups, makes that 10.4 (8.2 where the
// operands are in the Infinity Cache): neither launch has a workgroup for each of the 256 compute units.
constexpr int NORM_BACK_WAVES = 8;
constexpr int norm_back_threads(int T) { return T > 64 ? T : 64 * NORM_BACK_WAVES; }
constexpr int norm_back_rows(int T) { return T > 64 ? 1 : norm_back_threads(T) / T; }

template <int T, int NV, bool FP32>
__global__ __launch_bounds__(norm_back_threads(T)) void rms_norm_bwd(NormBackArgs a) {
    constexpr int ROWS = norm_back_rows(T), COLS = 8 * T * NV;
    static_assert(T > 64 || COLS <= 4 * norm_back_threads(T), "a thread for four columns");
    __shared__ float part[2][T > 64 ? T / 64 : 1];
    __shared__ __attribute__((aligned(16))) float meet[T <= 64 ? NORM_BACK_WAVES * COLS : 1];
    const int t = threadIdx.x % T, r = threadIdx.x / T;
    const int n = a.D >> 3;
    f32x8 sum[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[k][e] = 0.0f;
    int turn = 0;
    // the next row is on its way while this one is finished (4096 x 2048 bf16 20.4 us without, 18.2; 2048 x 8192 40.7, 34.1)
    f32x8 dy[NV];
    typedef typename std::conditional<FP32, f32x8, u32x4>::type Raw;
    Raw hv[NV];
    float next_rstd;
    auto load_raw = [&](const void* base, int64_t at, Raw& v) {
        if constexpr (FP32) load8(static_cast<const float*>(base) + at, v);
        else v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
    };
    auto fetch = [&](int64_t row) {
        next_rstd = a.rstd[row];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t + k * T;
            if (c >= n) continue;
            load8(a.dY + row * a.lddy + 8 * c, dy[k]);
            load_raw(a.h, row * a.ldh + 8 * c, hv[k]);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * ROWS + r, stride = (int64_t)gridDim.x * ROWS;
    if (first < a.B) fetch(first);
    for (int64_t row = first; row < a.B; row += stride) {
        f32x8 gy[NV], xh[NV];
        const float rstd = next_rstd;
        float dot = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t + k * T;
            if (c >= n) continue;
            f32x8 g;
            load8(a.gamma + 8 * c, g);
            if constexpr (!FP32) unpack8(hv[k], xh[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (FP32) xh[k][e] = hv[k][e];
                xh[k][e] *= rstd;
                sum[k][e] = fmaf(dy[k][e], xh[k][e], sum[k][e]);
                gy[k][e] = dy[k][e] * g[e];
                dot = fmaf(gy[k][e], xh[k][e], dot);
            }
        }
        Raw through[NV];                                       // before the next row's loads: they return in order
        if (a.dres != nullptr)
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (t + k * T < n) load_raw(a.dres, row * a.ldd + 8 * (t + k * T), through[k]);
        if (row + stride < a.B) fetch(row + stride);
        dot = row_sum<T>(dot, part[turn]) / (float)a.D;
        turn ^= 1;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t + k * T;
            if (c >= n) continue;
            f32x8 d;
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-dot, xh[k][e], gy[k][e]);
            if (a.dres != nullptr) {
                f32x8 more;
                if constexpr (!FP32) unpack8(through[k], more);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (FP32) more[e] = through[k][e];
                    d[e] += more[e];
                }
            }
            store_stream<FP32>(a.dh, row * a.lddh + 8 * c, d);
        }
    }
    if (a.parts == nullptr) return;
    if constexpr (T <= 64) {             // rows that share a wave, then the waves' shares, each thread four columns of all of them
#pragma unroll
        for (int m = T; m < 64; m <<= 1)
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[k][e] += __shfl_xor(sum[k][e], m, 64);
        if ((threadIdx.x & 63) < T)
#pragma unroll
            for (int k = 0; k < NV; ++k) store8(meet + (threadIdx.x >> 6) * COLS + 8 * (T * k + t), sum[k]);
        __syncthreads();
        const int c = 4 * threadIdx.x;
        if (c < a.D) {
            f32x4 v = *reinterpret_cast<const f32x4*>(meet + c);
#pragma unroll
            for (int w = 1; w < NORM_BACK_WAVES; ++w) v += *reinterpret_cast<const f32x4*>(meet + w * COLS + c);
            *reinterpret_cast<f32x4*>(a.parts + (int64_t)blockIdx.x * a.D + c) = v;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t + k * T;
            if (c < n) store8(a.parts + (int64_t)blockIdx.x * a.D + 8 * c, sum[k]);
        }
    }
}

// dgamma[d] = sum of the workgroups' shares, 32 columns to a workgroup: thread (q, c) sums four columns of shares q, q + 32, .., then the 32 sums
// of a column are added in their order.
__global__ __launch_bounds__(256) void rms_norm_dgamma(const float* __restrict__ parts, int n, int D, float* __restrict__ dgamma) {
    __shared__ float meet[32][36];
    const int c = threadIdx.x & 7, q = threadIdx.x >> 3;
    const f32x4* from = reinterpret_cast<const f32x4*>(parts + blockIdx.x * 32 + 4 * c);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int p = q; p < n; p += 32) s += from[(int64_t)p * (D / 4)];
    *reinterpret_cast<f32x4*>(&meet[q][4 * c]) = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        float v = meet[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < 32; ++w) v += meet[w][threadIdx.x];
        dgamma[blockIdx.x * 32 + threadIdx.x] = v;
    }
}

// Workgroups of the backward call: each leaves a share of dgamma that has to be written and read again.
static int norm_back_groups(int B, int D) {
    const int rows = norm_back_rows(D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : D <= 2048 ? 64 : 256), most = D <= 2048 ? 256 : 512;
    const int groups = (B + rows - 1) / rows;
    return groups < most ? groups : most;
}

static inline bool al(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// What both forward calls check, and their common arguments.
static int check_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int32_t stream_bytes, const float* gamma, float eps,
                      int32_t B, int32_t D, void* h, int64_t ldh, const void* y, int64_t ldy, const float* rstd) {
    if (!x || !gamma || !y) return WS_ERR_NULL;
    if (B <= 0 || D <= 0 || D % 64 || D > NORM_MAX_D || (stream_bytes != 2 && stream_bytes != 4)) return WS_ERR_SHAPE;
    if (ldx < D || (residual && ldr < D) || (h && ldh < D) || ldy < D) return WS_ERR_SHAPE;
    if (!(eps > 0.0f) || isinf(eps)) return WS_ERR_RANGE;
    const int unit = 16 / stream_bytes;
    if (!al(x, 16) || ldx % 8 || !al(gamma, 16) || !al(y, 16)) return WS_ERR_ALIGN;
    if ((residual && (!al(residual, 16) || ldr % unit)) || (h && (!al(h, 16) || ldh % unit))) return WS_ERR_ALIGN;
    if (rstd && !al(rstd, 4)) return WS_ERR_ALIGN;
    return WS_OK;
}

// A launch counts its threads with 32 bits, up to 1024 for a row: more rows go slice by slice.
constexpr int NORM_SLICE = 1 << 21;

template <bool FP32, bool MX>
static void launch_norm(NormArgs a, hipStream_t s) {
    for (int left = a.B; left > 0; left -= NORM_SLICE) {
        a.B = left < NORM_SLICE ? left : NORM_SLICE;
        if (a.D <= 64) hipLaunchKernelGGL((rms_norm_fwd<8, 1, FP32, MX>), dim3((a.B + 31) / 32), dim3(256), 0, s, a);
        else if (a.D <= 128) hipLaunchKernelGGL((rms_norm_fwd<16, 1, FP32, MX>), dim3((a.B + 15) / 16), dim3(256), 0, s, a);
        else if (a.D <= 256) hipLaunchKernelGGL((rms_norm_fwd<32, 1, FP32, MX>), dim3((a.B + 7) / 8), dim3(256), 0, s, a);
        else if (a.D <= 512) hipLaunchKernelGGL((rms_norm_fwd<64, 1, FP32, MX>), dim3((a.B + 3) / 4), dim3(256), 0, s, a);
        else if (a.D <= 1024) hipLaunchKernelGGL((rms_norm_fwd<64, 2, FP32, MX>), dim3((a.B + 3) / 4), dim3(256), 0, s, a);
        else if (a.D <= 2048) hipLaunchKernelGGL((rms_norm_fwd<64, 4, FP32, MX>), dim3((a.B + 3) / 4), dim3(256), 0, s, a);
        else if (a.D <= 4096) hipLaunchKernelGGL((rms_norm_fwd<256, 2, FP32, MX>), dim3(a.B), dim3(256), 0, s, a);
        else if (a.D <= 8192) hipLaunchKernelGGL((rms_norm_fwd<256, 4, FP32, MX>), dim3(a.B), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((rms_norm_fwd<1024, 2, FP32, MX>), dim3(a.B), dim3(1024), 0, s, a);
        a.x += a.B * a.ldx;
        if (a.res) a.res = static_cast<const char*>(a.res) + a.B * a.ldr * (FP32 ? 4 : 2);
        if (a.h) a.h = static_cast<char*>(a.h) + a.B * a.ldh * (FP32 ? 4 : 2);
        a.y = static_cast<char*>(a.y) + a.B * a.ldy * (MX ? 1 : 2);
        if (MX) a.scales += a.B * a.lds;
        if (a.rstd) a.rstd += a.B;
    }
}

template <bool FP32>
static void launch_norm_back(const NormBackArgs& a, int groups, hipStream_t s) {
    if (a.D <= 64) hipLaunchKernelGGL((rms_norm_bwd<8, 1, FP32>), dim3(groups), dim3(norm_back_threads(8)), 0, s, a);
    else if (a.D <= 128) hipLaunchKernelGGL((rms_norm_bwd<16, 1, FP32>), dim3(groups), dim3(norm_back_threads(16)), 0, s, a);
    else if (a.D <= 256) hipLaunchKernelGGL((rms_norm_bwd<32, 1, FP32>), dim3(groups), dim3(norm_back_threads(32)), 0, s, a);
    else if (a.D <= 512) hipLaunchKernelGGL((rms_norm_bwd<64, 1, FP32>), dim3(groups), dim3(norm_back_threads(64)), 0, s, a);
    else if (a.D <= 1024) hipLaunchKernelGGL((rms_norm_bwd<64, 2, FP32>), dim3(groups), dim3(norm_back_threads(64)), 0, s, a);
    else if (a.D <= 2048) hipLaunchKernelGGL((rms_norm_bwd<64, 4, FP32>), dim3(groups), dim3(norm_back_threads(64)), 0, s, a);
    else if (a.D <= 4096) hipLaunchKernelGGL((rms_norm_bwd<256, 2, FP32>), dim3(groups), dim3(256), 0, s, a);
    else if (a.D <= 8192) hipLaunchKernelGGL((rms_norm_bwd<256, 4, FP32>), dim3(groups), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rms_norm_bwd<1024, 2, FP32>), dim3(groups), dim3(1024), 0, s, a);
}

}  // namespace ws

using namespace ws;

extern "C" {

int ws_rms_norm_fwd(const void* x, int64_t ldx, const void* residual, int64_t ldr, int32_t stream_bytes, const float* gamma, float eps,
                    int32_t B, int32_t D, void* h, int64_t ldh, void* y, int64_t ldy, float* rstd, void* stream) {
    const int st = check_norm(x, ldx, residual, ldr, stream_bytes, gamma, eps, B, D, h, ldh, y, ldy, rstd);
    if (st != WS_OK) return st;
    if (ldy % 8) return WS_ERR_ALIGN;
    const NormArgs a = {static_cast<const uint16_t*>(x), ldx, residual, ldr, gamma, eps, B, D, h, ldh, y, ldy, nullptr, 0, rstd};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (stream_bytes == 4) launch_norm<true, false>(a, s);
    else launch_norm<false, false>(a, s);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

int ws_rms_norm_fwd_mx8(const void* x, int64_t ldx, const void* residual, int64_t ldr, int32_t stream_bytes, const float* gamma, float eps,
                        int32_t B, int32_t D, void* h, int64_t ldh, void* y, int64_t ldy, void* y_scales, int64_t lds, float* rstd,
                        void* stream) {
    if (!y_scales) return WS_ERR_NULL;
    const int st = check_norm(x, ldx, residual, ldr, stream_bytes, gamma, eps, B, D, h, ldh, y, ldy, rstd);
    if (st != WS_OK) return st;
    if (lds < D / MX_GROUP) return WS_ERR_SHAPE;
    if (ldy % 16 || !al(y_scales, 2) || lds % 2) return WS_ERR_ALIGN;
    const NormArgs a = {static_cast<const uint16_t*>(x), ldx, residual, ldr, gamma, eps, B, D, h, ldh, y, ldy,
                        static_cast<uint8_t*>(y_scales), lds, rstd};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (stream_bytes == 4) launch_norm<true, true>(a, s);
    else launch_norm<false, true>(a, s);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

size_t ws_rms_norm_bwd_workspace_bytes(int32_t B, int32_t D) {
    if (B <= 0 || D <= 0 || D % 64 || D > NORM_MAX_D) return 0;
    return (size_t)norm_back_groups(B, D) * D * 4;
}

int ws_rms_norm_bwd(const float* dY, int64_t lddy, const void* h, int64_t ldh, const void* dres, int64_t ldd, int32_t stream_bytes,
                    const float* gamma, const float* rstd, int32_t B, int32_t D, void* dh, int64_t lddh, float* dgamma,
                    void* workspace, size_t workspace_bytes, void* stream) {
    if (!dY || !h || !gamma || !rstd || !dh) return WS_ERR_NULL;
    if (B <= 0 || D <= 0 || D % 64 || D > NORM_MAX_D || (stream_bytes != 2 && stream_bytes != 4)) return WS_ERR_SHAPE;
    if (lddy < D || ldh < D || (dres && ldd < D) || lddh < D) return WS_ERR_SHAPE;
    const int unit = 16 / stream_bytes;
    if (!al(dY, 16) || lddy % 4 || !al(h, 16) || ldh % unit || !al(gamma, 16) || !al(rstd, 4) || !al(dh, 16) || lddh % unit) return WS_ERR_ALIGN;
    if ((dres && (!al(dres, 16) || ldd % unit)) || (dgamma && !al(dgamma, 4))) return WS_ERR_ALIGN;
    if (dgamma && (!workspace || workspace_bytes < ws_rms_norm_bwd_workspace_bytes(B, D))) return WS_ERR_WORKSPACE;
    if (dgamma && !al(workspace, 16)) return WS_ERR_ALIGN;
    const int groups = norm_back_groups(B, D);
    const NormBackArgs a = {dY, lddy, h, ldh, dres, ldd, gamma, rstd, B, D, dh, lddh, dgamma ? static_cast<float*>(workspace) : nullptr};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (stream_bytes == 4) launch_norm_back<true>(a, groups, s);
    else launch_norm_back<false>(a, groups, s);
    if (dgamma) hipLaunchKernelGGL(rms_norm_dgamma, dim3(D / 32), dim3(256), 0, s, a.parts, groups, D, dgamma);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

}  // extern "C"
