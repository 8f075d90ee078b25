// The split layer with 4-bit weights, for serving: logits and arg-max of a batch of tokens, and the packing of the weights.
//   z[i][c] = sum_d X[i][d] * W[c][d] + b[c],  W[c][d] = e2m1 code * 2^(scale byte of (c, d / 32) - 127)
// A batch of tokens reads every weight once and does two flops per token with it, so what bounds it is reading W: half a byte and
// 1/64 of the scale's byte per weight instead of bf16's two.
//
// The products run on the bf16 matrix instructions.  A code times its power of two is exact in bf16, and so is an e4m3 feature times
// its own, so only the fp32 sums round.  (The matrix instructions for 8- and 4-bit operands align the products of a group to the largest and
// drop what falls below: 4e-6 of the result's 2-norm at D = 2048 on normal data, where this path was exact; their rate is
// of no use while the weights' bytes bound the call.)
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/whalesplit.h"
#include "mx.h"

namespace ws {

// ---- packing ---------------------------------------------------------------------------------------------------------
// A thread takes eight neighbouring weights, four threads a group.  Ties round to the code with an even fraction bit.
__global__ __launch_bounds__(256) void quantize_mx4(const uint16_t* __restrict__ W, int64_t ldw, int64_t units, int per_row, uint8_t* __restrict__ W4,
                                                    int64_t ldw4, uint8_t* __restrict__ scales, int64_t lds) {
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / per_row;
        const int c = (int)(u - row * per_row);
        const u32x4 w = *reinterpret_cast<const u32x4*>(W + row * ldw + 8 * c);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = (w[e] & 0x7fffu) << 16, hi = w[e] & 0x7fff0000u;
            top = top > lo ? top : lo;
            top = top > hi ? top : hi;
        }
        const uint32_t byte = group_scale<E2M1_TOP_EXPONENT, E2M1_TOP_FRACTION>(quad_max(top));
        const float inv = inverse_scale(byte);
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(w[0] << 16) * inv, __uint_as_float(w[0] & 0xffff0000u) * inv, 1.0f, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(w[1] << 16) * inv, __uint_as_float(w[1] & 0xffff0000u) * inv, 1.0f, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(w[2] << 16) * inv, __uint_as_float(w[2] & 0xffff0000u) * inv, 1.0f, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(w[3] << 16) * inv, __uint_as_float(w[3] & 0xffff0000u) * inv, 1.0f, 3);
        *reinterpret_cast<uint32_t*>(W4 + row * ldw4 + 4 * c) = q;
        if ((c & 3) == 0) scales[row * lds + (c >> 2)] = (uint8_t)byte;
    }
}

// ---- products --------------------------------------------------------------------------------------------------------
struct W4Args {
    const uint8_t* X; int64_t ldx;           // bytes between rows
    const uint8_t* xs; int64_t ldxs;         // scales of e4m3 features, or nullptr: bf16
    const uint8_t* W; int64_t ldw;           // bytes between rows
    const uint8_t* ws; int64_t lds;
    const float* bias;
    int B, D, C;
    float* Z; int64_t ldz;
    float* part_val; int* part_cls; int class_offset;
};

constexpr int W4_SPAN = 512;                 // features that the lanes of a wave cover with four pieces of 32 each
constexpr int W4_WAVES = 4;
constexpr int W4_MAX_ROWS = WS_W4_MAX_ROWS;  // row tiles are counted in the grid's second extent

// A wave takes CT x 16 classes and NT x 16 rows.  Lane l holds class l % 16 (and row l % 16); of every span of 512 features it
// takes the 128 from 128 (l / 16) on, 32 at a time: 16 bytes of weights, whose four scales are neighbours.  Which features a matrix
// instruction sums over is free as long as both operands agree.
template <int NT, int CT, bool MX, bool TOP1>
__global__ __launch_bounds__(64 * W4_WAVES) void w4_product(W4Args a, int chunk, int groups) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int R = 16 * NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, g = lane >> 4;
    const int row0 = blockIdx.y * R;
    const int rows = a.B - row0 < R ? a.B - row0 : R;
    const int pitch = 2 * chunk + 16;
    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = lds + (16 * n + i16 < rows ? 16 * n + i16 : rows - 1) * pitch + 256 * g;
    float best[NT];
    int best_at[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        best[n] = -INFINITY;
        best_at[n] = INT_MAX;
    }

  for (int group = blockIdx.x; group < groups; group += gridDim.x) {
    const int class0 = (group * W4_WAVES + wave) * 16 * CT;
    // classes beyond the shard and rows beyond the batch repeat the last one: nothing of them is kept
    const uint8_t* w[CT];
    const uint8_t* ws[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int cls = class0 + 16 * c + i16;
        const int64_t at = cls < a.C ? cls : a.C - 1;
        w[c] = a.W + at * a.ldw + 64 * g;
        ws[c] = a.ws + at * a.lds + 4 * g;
    }
    f32x4 acc[CT][NT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[c][n] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int k0 = 0; k0 < a.D; k0 += chunk) {
        const int valid = a.D - k0 < chunk ? a.D - k0 : chunk;                 // a multiple of 64
        const int wide = (valid + W4_SPAN - 1) / W4_SPAN * W4_SPAN;            // zeros behind: weights that are not there count nothing
        __syncthreads();                                                       // the chunk before has been read
        const int units = wide >> 4;                                           // 16 features
        for (int u = tid; u < rows * units; u += 64 * W4_WAVES) {
            const int r = u / units, c = u - r * units;
            u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
            if (16 * c < valid) {
                const int64_t row = row0 + r;
                if constexpr (MX) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(a.X + row * a.ldx + k0 + 16 * c);
                    const float s = scale_of(a.xs[row * a.ldxs + (k0 >> 5) + (c >> 1)], 0);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        lo[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e], s, false));
                        lo[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e], s, true));
                        hi[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 + e], s, false));
                        hi[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 + e], s, true));
                    }
                } else {
                    const u32x4* p = reinterpret_cast<const u32x4*>(a.X + row * a.ldx + 2 * k0 + 32 * c);
                    lo = p[0];
                    hi = p[1];
                }
            }
            u32x4* q = reinterpret_cast<u32x4*>(lds + r * pitch + 32 * c);
            q[0] = lo;
            q[1] = hi;
        }
        __syncthreads();
        for (int s = 0; s < valid; s += W4_SPAN) {
            const int mine = a.D - k0 - s - 128 * g;                           // features from the lane's first on
            u32x4 v[CT][4];
            uint32_t sc[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const uint8_t* p = w[c] + ((k0 + s) >> 1);
                const uint8_t* ps = ws[c] + ((k0 + s) >> 5);
                sc[c] = 0;
                if (mine > 0) sc[c] = *reinterpret_cast<const uint16_t*>(ps);
                if (mine > 64) sc[c] |= (uint32_t)*reinterpret_cast<const uint16_t*>(ps + 2) << 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[c][i] = u32x4{0, 0, 0, 0};
                    if (mine > 32 * i) v[c][i] = *reinterpret_cast<const u32x4*>(p + 16 * i);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (s + 32 * i >= valid) break;                                // no lane has features there
                float f[CT];
#pragma unroll
                for (int c = 0; c < CT; ++c) f[c] = scale_of(sc[c], i);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16x8 wa[CT];
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        const uint32_t codes = v[c][i][q];
                        u32x4 t;
                        t[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f[c], 0));
                        t[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f[c], 1));
                        t[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f[c], 2));
                        t[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f[c], 3));
                        wa[c] = __builtin_bit_cast(bf16x8, t);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const bf16x8 xb = *reinterpret_cast<const bf16x8*>(x[n] + 2 * s + 64 * i + 16 * q);
#pragma unroll
                        for (int c = 0; c < CT; ++c) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[c], xb, acc[c][n], 0, 0, 0);
                    }
                }
            }
        }
    }

    // a lane holds four neighbouring classes of a row
    if constexpr (!TOP1) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int cls = class0 + 16 * c + 4 * g;
            f32x4 b = {0.f, 0.f, 0.f, 0.f};
            if (a.bias != nullptr)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (cls + e < a.C) b[e] = a.bias[cls + e];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = 16 * n + i16;
                if (r >= rows) continue;
                float* z = a.Z + (int64_t)(row0 + r) * a.ldz + cls;
                const f32x4 v = acc[c][n] + b;
                if (cls + 4 <= a.C) {
                    *reinterpret_cast<f32x4*>(z) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (cls + e < a.C) z[e] = v[e];
                }
            }
        }
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int cls = class0 + 16 * c + 4 * g + e;
                    if (cls < a.C) better_of(best[n], best_at[n], acc[c][n][e] + (a.bias != nullptr ? a.bias[cls] : 0.0f), cls);
                }
    }
  }
    if constexpr (TOP1) {
        __syncthreads();                                                       // the features have been read
        float* sv = reinterpret_cast<float*>(lds);
        int* sc = reinterpret_cast<int*>(sv + W4_WAVES * R);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            better_of(best[n], best_at[n], __shfl_xor(best[n], 16, 64), __shfl_xor(best_at[n], 16, 64));
            better_of(best[n], best_at[n], __shfl_xor(best[n], 32, 64), __shfl_xor(best_at[n], 32, 64));
            if (g == 0) {
                sv[wave * R + 16 * n + i16] = best[n];
                sc[wave * R + 16 * n + i16] = best_at[n];
            }
        }
        __syncthreads();
        if (tid < rows) {
            float v = sv[tid];
            int at = sc[tid];
#pragma unroll
            for (int k = 1; k < W4_WAVES; ++k) better_of(v, at, sv[k * R + tid], sc[k * R + tid]);
            a.part_val[(int64_t)blockIdx.x * a.B + row0 + tid] = v;
            a.part_cls[(int64_t)blockIdx.x * a.B + row0 + tid] = at == INT_MAX ? at : at + a.class_offset;
        }
    }
}

static inline bool al(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

static int w4_row_tiles(int B) { return B <= 16 ? 1 : B <= 32 ? 2 : 4; }
static int w4_groups(int C) { return (C + 63) / 64; }                          // of classes that a workgroup takes at a time
// Workgroups along the classes of the arg-max, each with a candidate for every row; they walk the groups.
constexpr int W4_MAX_PARTS = 4096;
static int w4_parts(int C) { return w4_groups(C) < W4_MAX_PARTS ? w4_groups(C) : W4_MAX_PARTS; }

template <int NT, bool MX, bool TOP1>
static void launch_w4_tiles(const W4Args& a, hipStream_t s) {
    const int most = NT == 1 ? 1536 : NT == 2 ? 512 : 512;
    const int chunk = a.D < most ? (a.D + W4_SPAN - 1) / W4_SPAN * W4_SPAN : most;
    const int rows = a.B < 16 * NT ? a.B : 16 * NT;
    size_t bytes = (size_t)rows * (2 * chunk + 16);
    const size_t least = TOP1 ? (size_t)W4_WAVES * 16 * NT * 8 : 0;
    if (bytes < least) bytes = least;
    hipLaunchKernelGGL((w4_product<NT, 1, MX, TOP1>), dim3(TOP1 ? w4_parts(a.C) : w4_groups(a.C), (a.B + 16 * NT - 1) / (16 * NT)),
                       dim3(64 * W4_WAVES), bytes, s, a, chunk, w4_groups(a.C));
}

template <bool TOP1>
static void launch_w4(const W4Args& a, hipStream_t s) {
    const int nt = w4_row_tiles(a.B);
    if (a.xs != nullptr) {
        if (nt == 1) launch_w4_tiles<1, true, TOP1>(a, s);
        else if (nt == 2) launch_w4_tiles<2, true, TOP1>(a, s);
        else launch_w4_tiles<4, true, TOP1>(a, s);
    } else {
        if (nt == 1) launch_w4_tiles<1, false, TOP1>(a, s);
        else if (nt == 2) launch_w4_tiles<2, false, TOP1>(a, s);
        else launch_w4_tiles<4, false, TOP1>(a, s);
    }
}

static int check_w4(const void* X, int64_t ldx, const void* X_scales, int64_t ldxs, const void* W4, int64_t ldw4, const void* W_scales,
                    int64_t lds, const float* b_shard, int32_t B, int32_t D, int32_t C_shard) {
    if (!X || !W4 || !W_scales) return WS_ERR_NULL;
    if (B <= 0 || D <= 0 || C_shard <= 0 || D % 64 || B > W4_MAX_ROWS) return WS_ERR_SHAPE;
    if (C_shard > INT32_MAX - 4096) return WS_ERR_RANGE;                       // class ids of a whole last group are counted in 31 bits
    if (ldx < D || (X_scales && ldxs < D / MX_GROUP) || ldw4 < D / 2 || lds < D / MX_GROUP) return WS_ERR_SHAPE;
    if (!al(X, 16) || ldx % (X_scales ? 16 : 8) || !al(W4, 16) || ldw4 % 16 || !al(W_scales, 2) || lds % 2) return WS_ERR_ALIGN;
    if ((X_scales && (!al(X_scales, 2) || ldxs % 2)) || (b_shard && !al(b_shard, 4))) return WS_ERR_ALIGN;
    return WS_OK;
}

static W4Args w4_args(const void* X, int64_t ldx, const void* X_scales, int64_t ldxs, const void* W4, int64_t ldw4, const void* W_scales,
                      int64_t lds, const float* b_shard, int32_t B, int32_t D, int32_t C_shard) {
    W4Args a = {};
    a.X = static_cast<const uint8_t*>(X); a.ldx = X_scales ? ldx : 2 * ldx;
    a.xs = static_cast<const uint8_t*>(X_scales); a.ldxs = ldxs;
    a.W = static_cast<const uint8_t*>(W4); a.ldw = ldw4;
    a.ws = static_cast<const uint8_t*>(W_scales); a.lds = lds;
    a.bias = b_shard;
    a.B = B; a.D = D; a.C = C_shard;
    return a;
}

}  // namespace ws

using namespace ws;

extern "C" {

int ws_quantize_mx4(const void* W, int64_t ldw, int32_t C, int32_t D, void* W4, int64_t ldw4, void* W_scales, int64_t lds, void* stream) {
    if (!W || !W4 || !W_scales) return WS_ERR_NULL;
    if (C <= 0 || D <= 0 || D % 64) return WS_ERR_SHAPE;
    if (ldw < D || ldw4 < D / 2 || lds < D / MX_GROUP) return WS_ERR_SHAPE;
    if (!al(W, 16) || ldw % 8 || !al(W4, 16) || ldw4 % 16 || !al(W_scales, 2) || lds % 2) return WS_ERR_ALIGN;
    const int64_t units = (int64_t)C * (D / 8);
    const int64_t groups = (units + 255) / 256;
    hipLaunchKernelGGL(quantize_mx4, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<const uint16_t*>(W), ldw, units, D / 8, static_cast<uint8_t*>(W4), ldw4, static_cast<uint8_t*>(W_scales), lds);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

int ws_split_fc_w4_logits(const void* X, int64_t ldx, const void* X_scales, int64_t ldxs, const void* W4, int64_t ldw4, const void* W_scales,
                          int64_t lds, const float* b_shard, int32_t B, int32_t D, int32_t C_shard, float* Z, int64_t ldz, void* stream) {
    if (!Z) return WS_ERR_NULL;
    const int st = check_w4(X, ldx, X_scales, ldxs, W4, ldw4, W_scales, lds, b_shard, B, D, C_shard);
    if (st != WS_OK) return st;
    if (ldz < C_shard) return WS_ERR_SHAPE;
    if (!al(Z, 16) || ldz % 4) return WS_ERR_ALIGN;
    W4Args a = w4_args(X, ldx, X_scales, ldxs, W4, ldw4, W_scales, lds, b_shard, B, D, C_shard);
    a.Z = Z; a.ldz = ldz;
    launch_w4<false>(a, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

size_t ws_w4_top1_workspace_bytes(int32_t B, int32_t C_shard) {
    return B > 0 && C_shard > 0 ? (size_t)w4_parts(C_shard) * B * 8 : 0;
}

int ws_split_fc_w4_top1(const void* X, int64_t ldx, const void* X_scales, int64_t ldxs, const void* W4, int64_t ldw4, const void* W_scales,
                        int64_t lds, const float* b_shard, int32_t B, int32_t D, int32_t C_shard, int32_t class_offset, float* top_logit,
                        int32_t* top_class, void* workspace, size_t workspace_bytes, void* stream) {
    if (!top_logit || !top_class) return WS_ERR_NULL;
    const int st = check_w4(X, ldx, X_scales, ldxs, W4, ldw4, W_scales, lds, b_shard, B, D, C_shard);
    if (st != WS_OK) return st;
    if (class_offset < 0 || (int64_t)class_offset + C_shard > INT32_MAX) return WS_ERR_RANGE;
    if (!al(top_logit, 4) || !al(top_class, 4)) return WS_ERR_ALIGN;
    if (!workspace || workspace_bytes < ws_w4_top1_workspace_bytes(B, C_shard)) return WS_ERR_WORKSPACE;
    if (!al(workspace, 16)) return WS_ERR_ALIGN;
    W4Args a = w4_args(X, ldx, X_scales, ldxs, W4, ldw4, W_scales, lds, b_shard, B, D, C_shard);
    const int parts = w4_parts(C_shard);
    a.part_val = static_cast<float*>(workspace);
    a.part_cls = reinterpret_cast<int*>(a.part_val + (int64_t)parts * B);
    a.class_offset = class_offset;
    launch_w4<true>(a, static_cast<hipStream_t>(stream));
    if (hipGetLastError() != hipSuccess) return WS_ERR_HIP;
    return ws_combine_top1(a.part_val, a.part_cls, parts, B, B, top_logit, top_class, stream);
}

}  // extern "C"
