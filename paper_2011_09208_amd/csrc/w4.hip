// The split layer with 4-bit weights, for serving: logits and arg-max of a batch of tokens, and the packing of the weights.
//   z[i][c] = sum_d X[i][d] * W[c][d] + b[c],  W[c][d] = e2m1 code * 2^(scale byte of (c, d / 32) - 127)
// A batch of tokens reads every weight once and does two flops per token with it, so what bounds it is reading W: half a byte
// of code and 1/32 of a byte of scale per weight instead of bf16's two.
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
#include "w4_plan.h"

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
    float* part_val; int* part_cls;          // [B][workgroups along the classes]
};

// Where a lane loads and where its data goes.  A load takes 16 bytes of codes a lane, four neighbouring lanes 64 bytes of a class row: 16 rows x 64
// bytes, one step of 16 classes.  With a lane for each row, as the matrix instruction has them, every lane is in a cache line of its own and
// the addresses of a load take four times as long.  For the product lane l holds class l % 16 and the 32 features from 32 (l / 16) on, which
// the lanes fetch from each other; which features an instruction sums over is free as long as both operands agree.
struct W4Lane {
    int i16, g;                              // of the product: class (and row) and group of 32 features
    int seg;                                 // of a load: 16-byte piece of class row lane / 4
    int codes, scale;                        // byte offsets of the lanes to fetch from: codes, and the scales of step 0
    int turn;                                // brings scale byte g of a step's four to a float's exponent
    int code_offset, scale_offset;           // of a load, from the tile's first byte
    __device__ __forceinline__ W4Lane(int lane, const W4Args& a)
        : i16(lane & 15), g(lane >> 4), seg(lane & 3), codes(4 * (4 * (lane & 15) + (lane >> 4))), scale(16 * (lane & 15)),
          turn((8 * (lane >> 4) + 9) & 31), code_offset((lane >> 2) * (int)a.ldw + 16 * (lane & 3)), scale_offset((lane >> 2) * (int)a.lds) {}
};

// Sixteen class rows of codes and of scales as buffers: what lies beyond the last class reads as zeros, without a branch.  A branch around
// loads, even one that is never taken, makes the compiler wait for them as if nothing had been loaded since.  A step's first byte is the loads'
// scalar offset: a load is in range if lane offset + scalar offset lies within the buffer, as a sum that does not wrap (measured, make_operand), so the
// steps behind the last class's last feature read nothing.  (The first byte in the lanes' offsets spills registers in w4_tiles, and so does a buffer for
// each step.)
struct W4Tile {
    __amdgpu_buffer_rsrc_t codes, scales;
    // classes [cls, cls + 16) of the shard; none of them if cls >= C
    __device__ __forceinline__ W4Tile(const W4Args& a, int cls) {
        const int64_t n = a.C - cls < 16 ? a.C - cls : 16;
        const int64_t at = n > 0 ? cls : 0;
        const int code_bytes = n > 0 ? (int)((n - 1) * a.ldw + (a.D >> 1)) : 0, scale_bytes = n > 0 ? (int)((n - 1) * a.lds + (a.D >> 5)) : 0;
        codes = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.W + at * a.ldw), 0, code_bytes, 0x00020000);
        scales = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.ws + at * a.lds), 0, scale_bytes, 0x00020000);
    }
};

// Codes and scales of N steps of a tile; of the scales, lane l holds steps l % 4, l % 4 + 4, ..
template <int N> struct W4Piece {
    static constexpr int HELD = (N + 3) / 4;
    u32x4 v[N];
    uint16_t s[HELD], t[HELD];               // two scales each
};

// From feature k on (a step's first).  Beyond the row's end it may read the next row's bytes: codes stand for numbers whatever they are, and the
// features there are zeros; scales are masked when they are used.
template <int N>
__device__ __forceinline__ void w4_load(W4Piece<N>& p, const W4Tile& tile, const W4Lane& l, int k) {
#pragma unroll
    for (int i = 0; i < N; ++i) p.v[i] = __builtin_amdgcn_raw_buffer_load_b128(tile.codes, l.code_offset + 64 * i, k >> 1, 0);
#pragma unroll
    for (int j = 0; j < W4Piece<N>::HELD; ++j) {
        const int off = l.scale_offset + 4 * (N >= 4 ? 4 * j + l.seg : l.seg & (N - 1));
        p.s[j] = __builtin_amdgcn_raw_buffer_load_b16(tile.scales, off, k >> 5, 0);
        p.t[j] = __builtin_amdgcn_raw_buffer_load_b16(tile.scales, off + 2, k >> 5, 0);
    }
}

// The two halves of four scales.  In assembly: an ordinary expression is moved up to right behind the loads, and waits for them there.
template <int N>
__device__ __forceinline__ void w4_join(uint32_t (&joined)[W4Piece<N>::HELD], const W4Piece<N>& p) {
#pragma unroll
    for (int j = 0; j < W4Piece<N>::HELD; ++j)
        asm volatile("v_perm_b32 %0, %1, %2, %3" : "=v"(joined[j]) : "v"(p.t[j]), "v"(p.s[j]), "s"(0x05040100));
}

// The lane's codes and scale of step i for the product, of which `left` features from step 0 on are there (a multiple of 64).
template <int N>
__device__ __forceinline__ u32x4 w4_codes(const W4Piece<N>& p, int i, const W4Lane& l) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (uint32_t)__builtin_amdgcn_ds_bpermute(l.codes, (int)p.v[i][e]);
    return v;
}
template <bool WHOLE, int HELD>
__device__ __forceinline__ float w4_scale(const uint32_t (&joined)[HELD], int i, int left, const W4Lane& l) {
    const uint32_t four = (uint32_t)__builtin_amdgcn_ds_bpermute(l.scale + 4 * (i & 3), (int)joined[i >> 2]);
    const uint32_t f = __builtin_amdgcn_alignbit(four, four, l.turn);
    return __uint_as_float(WHOLE || W4_STEP * i + 32 * l.g < left ? f : 0u);
}

// Eight e4m3 values as bf16, times the scale.
__device__ __forceinline__ u32x4 w4_features(uint32_t a, uint32_t b, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true))};
}

// Features of rows [row0, row0 + rows), [k0, k0 + 128 steps), as bf16 into LDS: plane g of four holds the 32 features that lane group g
// reads of every step, [row][step] with a pitch of an odd number of 16-byte chunks, so that the 16 rows of a read differ in their banks (the
// planes are whole 256 bytes apart).  Zeros stand for features beyond D.
template <int THREADS, bool MX>
__device__ __forceinline__ void w4_stage(const W4Args& a, int row0, int rows, int k0, int steps, char* lds, int pitch, int plane) {
    const int units = steps * (W4_STEP / 16), left = a.D - k0;
    for (int u = threadIdx.x; u < rows * units; u += THREADS) {
        const int r = u / units, c = u - r * units;                            // 16 features from 16 c on
        u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        if (16 * c < left) {
            const int64_t row = row0 + r;
            if constexpr (MX) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(a.X + row * a.ldx + k0 + 16 * c);
                const float s = scale_of(a.xs[row * a.ldxs + (k0 >> 5) + (c >> 1)], 0);
                lo = w4_features(v[0], v[1], s);
                hi = w4_features(v[2], v[3], s);
            } else {
                const u32x4* p = reinterpret_cast<const u32x4*>(a.X + row * a.ldx + 2 * k0 + 32 * c);
                lo = p[0];
                hi = p[1];
            }
        }
        u32x4* q = reinterpret_cast<u32x4*>(lds + ((c >> 1) & 3) * plane + r * pitch + (c >> 3) * 64 + (c & 1) * 32);
        q[0] = lo;
        q[1] = hi;
    }
}

// Eight codes as bf16, times the scale.
__device__ __forceinline__ bf16x8 w4_values(uint32_t codes, float scale) {
    return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                                            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                                            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                                            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))});
}

// acc += codes x features of `left` (at most PIECE steps) features; x[n] points at the lane's row of its plane, at the piece's first step.
template <bool WHOLE, int CT, int PIECE, int NT>
__device__ __forceinline__ void w4_multiply_steps(f32x4 (&acc)[CT][NT], const W4Piece<PIECE> (&p)[CT], const char* const (&x)[NT], int at, int left,
                                                  const W4Lane& l) {
    uint32_t joined[CT][W4Piece<PIECE>::HELD];
#pragma unroll
    for (int c = 0; c < CT; ++c) w4_join(joined[c], p[c]);
#pragma unroll
    for (int i = 0; i < PIECE; ++i) {
        if (!WHOLE && W4_STEP * i >= left) break;
        float f[CT];
        u32x4 v[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            f[c] = w4_scale<WHOLE>(joined[c], i, left, l);
            v[c] = w4_codes(p[c], i, l);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 wa[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) wa[c] = w4_values(v[c][q], f[c]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bf16x8 xb = *reinterpret_cast<const bf16x8*>(x[n] + at + 64 * i + 16 * q);
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[c], xb, acc[c][n], 0, 0, 0);
            }
        }
    }
}
template <int CT, int PIECE, int NT>
__device__ __forceinline__ void w4_multiply(f32x4 (&acc)[CT][NT], const W4Piece<PIECE> (&p)[CT], const char* const (&x)[NT], int at, int left, const W4Lane& l) {
    if (left >= PIECE * W4_STEP) w4_multiply_steps<true>(acc, p, x, at, left, l);
    else w4_multiply_steps<false>(acc, p, x, at, left, l);
}

// The biases as a buffer, zeros without a bias and beyond the shard; four classes' from class cls on.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t w4_biases(const W4Args& a) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.bias), 0, a.bias != nullptr ? (int)(4u * (uint32_t)a.C) : 0, 0x00020000);
}
__device__ __forceinline__ f32x4 w4_bias(__amdgpu_buffer_rsrc_t biases, int cls) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(biases, (int)(4u * (uint32_t)cls), 0, 0));
}

// Four neighbouring logits, of which the first `n` (any number) are there.
__device__ __forceinline__ void w4_store(float* z, f32x4 v, int n) {
    if (n >= 4) {
        *reinterpret_cast<f32x4*>(z) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) z[e] = v[e];
    }
}

// The logits of four neighbouring classes of 16 NT rows: stored, or held against the best so far.
template <int NT, bool TOP1>
__device__ __forceinline__ void w4_finish(const W4Args& a, const f32x4 (&acc)[NT], f32x4 b, int cls, int row0, int rows, int i16, float* best,
                                          int* best_at) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const f32x4 v = acc[n] + b;
        if constexpr (TOP1) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (cls + e < a.C) better_of(best[n], best_at[n], v[e], cls + e);
        } else {
            const int r = 16 * n + i16;
            if (r >= rows) continue;
            w4_store(a.Z + (int64_t)(row0 + r) * a.ldz + cls, v, a.C - cls);
        }
    }
}

// The workgroup's candidates of its rows, out of its lanes' and waves'.
template <int NT, int WAVES>
__device__ __forceinline__ void w4_report(const W4Args& a, float (&best)[NT], int (&best_at)[NT], int row0, int rows, const W4Lane& l, char* lds, int part, int parts) {
    constexpr int R = 16 * NT;
    __syncthreads();                                                           // the features have been read
    float* sv = reinterpret_cast<float*>(lds);
    int* sc = reinterpret_cast<int*>(sv + WAVES * R);
    const int tid = threadIdx.x, wave = tid >> 6;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        better_of(best[n], best_at[n], __shfl_xor(best[n], 16, 64), __shfl_xor(best_at[n], 16, 64));
        better_of(best[n], best_at[n], __shfl_xor(best[n], 32, 64), __shfl_xor(best_at[n], 32, 64));
        if (l.g == 0) {
            sv[wave * R + 16 * n + l.i16] = best[n];
            sc[wave * R + 16 * n + l.i16] = best_at[n];
        }
    }
    __syncthreads();
    if (tid < rows) {
        float v = sv[tid];
        int at = sc[tid];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) better_of(v, at, sv[k * R + tid], sc[k * R + tid]);
        a.part_val[(int64_t)(row0 + tid) * parts + part] = v;
        a.part_cls[(int64_t)(row0 + tid) * parts + part] = at;
    }
}

// ---- many rows ---------------------------------------------------------------------------------------------------------
// A wave takes CT x 16 classes and 16 NT rows, a workgroup WAVES waves along the classes; tile c of all waves makes WAVES x 16 neighbouring classes.
// A step of the rows' features is in LDS, the next one on its way to the other half, and so are the next codes.  A step takes 2.2 us with 64
// rows, most of it the way of its codes: load, exchange between lanes, conversion, product; with 256 rows the matrix instructions and LDS, from which
// every wave reads every feature fragment, for CT products each.  201 x 1088 x 50 001: 38.5 us with
// codes and logits in HBM, 33.3 where the 69 MB that a call moves are in the Infinity Cache; 128 x 2048 x 100 000: 65 (800 TFLOP/s), 256: 123 (850).
// Up to 64 rows CT = 2 leaves registers for two workgroups on a compute unit, which fill each other's pauses (64 x 256 x 100 000 classes 15.2 us,
// CT = 4 17.8); with more rows CT = 4 halves what is read from LDS for a product.
//
// With four waves, where a compute unit has no second workgroup, two steps of codes and features are on their way (96 x 2048 x 12 500 18.7 us, now
// 17.8; 20 x 10 240 x 3000 61, 47).
//
// Tried and slower: the same with eight waves (64 x 2048 x 100 000 classes 48.8 us, now 47.4); the scales of 16 steps through LDS
// (a step of 64 rows is 15 % faster, but the start costs 7 us: 200 x 1088 x 50 001 49.6 us, 39.8 for the kernel of then without them).
//
// Logits leave through LDS, one c after the other, in a loop that is not unrolled: straight from the accumulators every one of the CT NT 4 stores
// and bounds checks is code of its own, 10 KiB that each launch fetches anew (128 rows x 256 features x 100 000 classes 28.6 us).
template <int NT, int CT, int WAVES, bool MX, bool TOP1>
__global__ __launch_bounds__(64 * WAVES, CT == 2 && WAVES == 8 ? 4 : 2) void w4_tiles(W4Args a, int groups, int row_blocks, int parts) {
    constexpr int R = 16 * NT, THREADS = 64 * WAVES, STRIP = 16 * WAVES, CLASSES = CT * STRIP;
    constexpr int PITCH = 64 + 16, PLANE = (R * PITCH + 255) & ~255, HALF = 4 * PLANE;
    constexpr int OUT_PITCH = STRIP + 4;                                           // floats
    constexpr int OUT_BYTES = R * OUT_PITCH * 4;
    constexpr int UNITS = (R * 8 + THREADS - 1) / THREADS;                         // of 16 features that a thread brings to LDS in a step
    constexpr bool EARLY = CT * NT <= 24;                                          // registers for the next step's codes in the product's order, too
    constexpr int SETS = WAVES == 4 ? 2 : 1;                                       // steps on their way
    __shared__ __attribute__((aligned(16))) char lds[2 * HALF > OUT_BYTES ? 2 * HALF : OUT_BYTES];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const W4Lane l(tid & 63, a);
    // the row blocks of a group of classes run on one XCD one after the other, and find its codes in that L2
    const int slot = blockIdx.x >> 3, block = slot % row_blocks, first = (blockIdx.x & 7) + 8 * (slot / row_blocks);
    if (first >= parts) return;
    const int row0 = block * R;
    const int rows = a.B - row0 < R ? a.B - row0 : R;
    const int steps = (a.D + W4_STEP - 1) / W4_STEP;
    const char* x = lds + l.g * PLANE + l.i16 * PITCH;                             // rows beyond the batch stay as LDS has them: nothing of them is kept
    const __amdgpu_buffer_rsrc_t biases = w4_biases(a);
    // in the output loop QUADS threads share a row, and a thread takes four classes of every PER-th row
    constexpr int QUADS = STRIP / 4, PER = THREADS / QUADS, TURNS = R / PER;
    static_assert(QUADS <= 64 && R % PER == 0, "");
    const int out_row = tid / QUADS, out_quad = tid % QUADS;
    float best[TOP1 ? TURNS : 1];
    int best_at[TOP1 ? TURNS : 1];
    if constexpr (TOP1)
#pragma unroll
        for (int j = 0; j < TURNS; ++j) {
            best[j] = -INFINITY;
            best_at[j] = INT_MAX;
        }

    // this thread's units of a step
    const uint8_t* from[UNITS];
    const uint8_t* from_scale[UNITS];
    int to[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int u = tid + THREADS * j, r = u >> 3, c = u & 7;
        const int64_t row = row0 + (r < rows ? r : rows - 1);
        from[j] = a.X + row * a.ldx + (MX ? 16 : 32) * c;
        from_scale[j] = MX ? a.xs + row * a.ldxs + (c >> 1) : nullptr;
        to[j] = r < rows ? ((c >> 1) & 3) * PLANE + r * PITCH + (c & 1) * 32 : -1;
    }
    struct Rows {
        u32x4 a[UNITS], b[UNITS];
        uint32_t s[UNITS];
    } coming[SETS];
    // No branch around the loads; beyond the row's end, half a step at most, the last features are loaded once more and zeros are staged.
    auto fetch = [&](Rows& w, int step) {
        const int s = step < steps ? step : steps - 1;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int c = (tid + THREADS * j) & 7;
            const int back = s * W4_STEP + 16 * c < a.D ? 0 : 64;
            const u32x4* p = reinterpret_cast<const u32x4*>(from[j] + (MX ? 1 : 2) * (s * W4_STEP - back));
            w.a[j] = p[0];
            if constexpr (MX) w.s[j] = from_scale[j][s * 4 - back / 32];
            else w.b[j] = p[1];
        }
    };
    auto stage = [&](const Rows& w, int step) {
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            if (to[j] < 0) continue;
            const int c = (tid + THREADS * j) & 7;
            u32x4 lo = w.a[j], hi = w.b[j];
            if constexpr (MX) {
                const float f = scale_of(w.s[j], 0);
                lo = w4_features(w.a[j][0], w.a[j][1], f);
                hi = w4_features(w.a[j][2], w.a[j][3], f);
            }
            if (step * W4_STEP + 16 * c >= a.D) lo = hi = u32x4{0, 0, 0, 0};
            u32x4* q = reinterpret_cast<u32x4*>(lds + (step & 1) * HALF + to[j]);
            q[0] = lo;
            q[1] = hi;
        }
    };

    for (int group = first; group < groups; group += parts) {
        const int class0 = group * CLASSES + wave * 16;
        W4Piece<1> codes[SETS][CT];
        auto load = [&](W4Piece<1> (&p)[CT], int step) {
#pragma unroll
            for (int c = 0; c < CT; ++c) w4_load(p[c], W4Tile(a, class0 + STRIP * c), l, step * W4_STEP);
        };
        float f[CT];                                                               // codes and scales in the product's order
        u32x4 v[CT];
        auto take = [&](float (&to_f)[CT], u32x4 (&to_v)[CT], const W4Piece<1> (&p)[CT], int c, int step) {
            uint32_t joined[1];
            w4_join(joined, p[c]);
            to_f[c] = w4_scale<false>(joined, 0, a.D - step * W4_STEP, l);
            to_v[c] = w4_codes(p[c], 0, l);
        };
        f32x4 acc[CT][NT];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[c][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        fetch(coming[0], 0);
        load(codes[0], 0);
        if constexpr (SETS == 2) {
            fetch(coming[1], 1);
            load(codes[1], 1);
        }
        stage(coming[0], 0);
        if constexpr (EARLY) {
#pragma unroll
            for (int c = 0; c < CT; ++c) take(f, v, codes[0], c, 0);
            load(codes[0], SETS);
        }
        wait_counts<NO_VM_WAIT, 0>();
        raw_barrier();
        // `p` holds the codes of this step, or of the next one if they are taken early; `free` and `next` are the rows' features behind the next step
        // and of it.  Loads return in order: features that came from the cache one step ahead would wait for the codes two steps ahead.
        auto turn = [&](W4Piece<1> (&p)[CT], Rows& free, const Rows& next, int step) {
            fetch(free, step + SETS);
            if constexpr (!EARLY) {
#pragma unroll
                for (int c = 0; c < CT; ++c) take(f, v, p, c, step);
                load(p, step + 1);
            }
            // Fragments of the features are read three ahead, and the codes of the next quarter of a step turned into values meanwhile; the order is
            // pinned, left alone the reads end up right in front of their products and the loads behind them.
            const char* at = x + (step & 1) * HALF;
            auto fragment = [&](int i) { return *reinterpret_cast<const bf16x8*>(at + 16 * PITCH * (i % NT) + 16 * (i / NT)); };
            bf16x8 ring[4], wa[CT], ahead[CT];
            float next_f[CT];
            u32x4 next_v[CT];
#pragma unroll
            for (int i = 0; i < 3; ++i) ring[i] = fragment(i);
#pragma unroll
            for (int c = 0; c < CT; ++c) wa[c] = w4_values(v[c][0], f[c]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4 * NT; ++i) {
                const int q = i / NT, n = i % NT;
                if (i + 3 < 4 * NT) ring[(i + 3) & 3] = fragment(i + 3);
                if (q < 3)
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        if (c % NT == n) ahead[c] = w4_values(v[c][q + 1], f[c]);
                if (EARLY && q >= 2)                                               // the next step's codes, a tile at a time in the second half of this one
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        if (c == (i - 2 * NT) * CT / (2 * NT) && (i == 2 * NT || c != (i - 1 - 2 * NT) * CT / (2 * NT))) take(next_f, next_v, p, c, step + 1);
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[c], ring[i & 3], acc[c][n], 0, 0, 0);
                if (n == NT - 1)
#pragma unroll
                    for (int c = 0; c < CT; ++c) wa[c] = ahead[c];
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (EARLY) {
                load(p, step + 1 + SETS);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    f[c] = next_f[c];
                    v[c] = next_v[c];
                }
            }
            stage(next, step + 1);
            wait_counts<NO_VM_WAIT, 0>();
            raw_barrier();                                                         // the codes stay in flight
        };
#pragma unroll 1
        for (int step = 0; step < steps; step += SETS)
#pragma unroll
            for (int i = 0; i < SETS; ++i)                                         // a step too many adds zeros
                turn(codes[EARLY ? (i + 1) % SETS : i], coming[i], coming[(i + 1) % SETS], step + i);
        float* out = reinterpret_cast<float*>(lds);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) *reinterpret_cast<f32x4*>(out + (16 * n + l.i16) * OUT_PITCH + 16 * wave + 4 * l.g) = acc[c][n];
            const int cls = group * CLASSES + STRIP * c + 4 * out_quad;
            const f32x4 bias = w4_bias(biases, cls);
            __syncthreads();
            if constexpr (TOP1) {
#pragma unroll
                for (int j = 0; j < TURNS; ++j) {
                    const f32x4 z = *reinterpret_cast<const f32x4*>(out + (out_row + j * PER) * OUT_PITCH + 4 * out_quad) + bias;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (cls + e < a.C) better_of(best[j], best_at[j], z[e], cls + e);
                }
            } else {
#pragma unroll 1
                for (int r = out_row; r < rows; r += PER) {
                    const f32x4 z = *reinterpret_cast<const f32x4*>(out + r * OUT_PITCH + 4 * out_quad) + bias;
                    w4_store(a.Z + (int64_t)(row0 + r) * a.ldz + cls, z, a.C - cls);
                }
            }
            __syncthreads();
        }
    }
    if constexpr (TOP1) {
#pragma unroll
        for (int j = 0; j < TURNS; ++j) {
            for (int m = 1; m < QUADS; m <<= 1) better_of(best[j], best_at[j], __shfl_xor(best[j], m, 64), __shfl_xor(best_at[j], m, 64));
            const int r = out_row + j * PER;
            if (out_quad == 0 && r < rows) {
                a.part_val[(int64_t)(row0 + r) * parts + first] = best[j];
                a.part_cls[(int64_t)(row0 + r) * parts + first] = best_at[j];
            }
        }
    }
}

// ---- few rows, many classes --------------------------------------------------------------------------------------------
// One workgroup to a compute unit holds all features of up to 16 NT rows in LDS.  Its 16 waves walk tiles of 16 classes, each by itself, with
// no barrier between them: a tile's codes are a stream of pieces of 512 features, RING of them loaded at a time.  With many tiles the waves'
// loads cover for each other and RING = 1 does: the code is short, and a kernel of a few us pays for every line of it (all kernels start with an
// empty instruction cache; 8 rows x 512 features x 2000 classes 3.2 us, RING = 2 4.8, 3 6.4).
constexpr int W4_STREAM_WAVES = 16, W4_STREAM_THREADS = 64 * W4_STREAM_WAVES;
constexpr int W4_STREAM_PIECE = 4;

template <int NT, int RING, bool MX, bool TOP1>
__global__ __launch_bounds__(W4_STREAM_THREADS) void w4_stream(W4Args a, int tiles) {
    constexpr int PIECE = W4_STREAM_PIECE, SPAN = PIECE * W4_STEP;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const W4Lane l(tid & 63, a);
    const int rows = a.B, steps = (a.D + W4_STEP - 1) / W4_STEP;
    const int pitch = 64 * steps + 16, plane = (rows * pitch + 255) & ~255;
    const int stride = gridDim.x * W4_STREAM_WAVES;

    // the piece that is loaded next; behind the last tile nothing is there
    int tile = wave * gridDim.x + blockIdx.x, k = 0;
    int now = tile, at = 0;                                                        // the piece that is multiplied
    W4Piece<PIECE> ring[RING][1];
    f32x4 bias[RING];                                                              // of the tile that ends with this piece
    W4Tile aim(a, 16 * tile);
    const __amdgpu_buffer_rsrc_t biases = w4_biases(a);
    auto load = [&](int i) {
        w4_load(ring[i][0], aim, l, k);
        k += SPAN;
        const bool last = k >= a.D;
        uint32_t from = 64u * (uint32_t)tile;                                      // no bias is fetched with the other pieces: beyond any buffer
        if (!last) from = 0u - 1024u;
        bias[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(biases, (int)(from + 16u * (uint32_t)l.g), 0, 0));
        if (last) {
            k = 0;
            tile = tile + stride < tiles ? tile + stride : tiles;
            aim = W4Tile(a, 16 * tile);
        }
    };
#pragma unroll
    for (int i = 0; i < RING; ++i) load(i);
    w4_stage<W4_STREAM_THREADS, MX>(a, 0, rows, 0, steps, lds, pitch, plane);
    __syncthreads();

    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = lds + l.g * plane + (16 * n + l.i16 < rows ? 16 * n + l.i16 : rows - 1) * pitch;
    float best[NT];
    int best_at[NT];
    f32x4 acc[1][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        best[n] = -INFINITY;
        best_at[n] = INT_MAX;
        acc[0][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    while (now < tiles) {
#pragma unroll
        for (int i = 0; i < RING; ++i) {                                           // pieces behind the last tile are zeros, and their classes beyond the shard
            w4_multiply<1, PIECE, NT>(acc, ring[i], x, at / 2, a.D - at, l);
            at += SPAN;
            if (at >= a.D) {
                const int cls = 16 * now + 4 * l.g;                                // a lane holds four neighbouring classes of a row
                w4_finish<NT, TOP1>(a, acc[0], bias[i], cls, 0, rows, l.i16, best, best_at);
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[0][n] = f32x4{0.f, 0.f, 0.f, 0.f};
                at = 0;
                now = now + stride < tiles ? now + stride : tiles;
            }
            load(i);
        }
    }
    if constexpr (TOP1) w4_report<NT, W4_STREAM_WAVES>(a, best, best_at, 0, rows, l, lds, blockIdx.x, gridDim.x);
}

// ---- few tiles of rows and classes -----------------------------------------------------------------------------------
// The waves of a workgroup share out the contraction, so that all codes of its classes are on their way at once, and the waves' partial sums
// meet in LDS.  One workgroup per group of classes, most of a compute unit's wave slots filled with them: reading alone, W of 100 000 x 2048
// takes 16.9 us so, 19.9 with a wave for 16 whole rows; 1000 x 4096 2.8 and 6.8.
//
// Wave k takes the steps S k .. S k + S - 1 of CT tiles of 16 classes.  Rows go 16 NT at a time, and P steps of them at a time through LDS, where
// each wave has a region of its own.  Up to 32 rows at a time: 32 x 2048 x 12 500 took 11.2 us in
// two halves, 64 18.5 in four.  Blocks of rows go side by side where units are free: 128 x 2048 x 3000 14.4 us one after the other, 7.9.
constexpr int W4_FEW_THREADS = 64 * W4_FEW_WAVES;
constexpr int w4_few_piece(int S, int CT, int NT, bool MX) { return S >= 2 && S <= 4 && (MX || CT * S * NT == 2) ? 2 : 1; }          // P, as many as the registers hold
constexpr int w4_few_plane(int P, int rows) { return (rows * (64 * P + 16) + 255) & ~255; }
constexpr int w4_few_region(int P, int CT, int rows) {
    const int features = 4 * w4_few_plane(P, rows), sums = rows * (16 * CT + 4) * 4;
    return features > sums ? features : (sums + 255) & ~255;
}

template <int S, int CT, int NT, bool MX, bool TOP1>
__global__ __launch_bounds__(W4_FEW_THREADS, S * CT * NT < 8 ? 4 : 2) void w4_few(W4Args a) {
    constexpr int P = w4_few_piece(S, CT, NT, MX), PITCH = 16 * CT + 4, R = 16 * NT;
    constexpr int UNITS = (MX ? P * 2 : P * 4) * NT;                               // 16-byte loads of a lane for a piece of R rows
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const W4Lane l(lane, a);
    const int i16 = l.i16, g = l.g;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int step0 = wave * S;
    const int row0 = blockIdx.y * R, stride = gridDim.y * R;
    const int most = a.B < R ? a.B : R;
    const int plane = w4_few_plane(P, most), region = w4_few_region(P, CT, most);
    char* mine = lds + wave * region;
    const int first = blockIdx.x * 16 * CT;                                        // the workgroup's first class
    // this thread's four neighbouring classes in the sum over the waves, of every (512 / QUADS)-th row
    constexpr int QUADS = 4 * CT;
    const int c4 = tid & (QUADS - 1);
    const int cls = first + 4 * c4;

    const f32x4 bias = w4_bias(w4_biases(a), cls);

    // features [8 u, 8 u + 8) (MX: 16) of a piece and row, as the lane's load j: u + units per row * row = lane + 64 j
    constexpr int ROW_UNITS = MX ? 8 * P : 16 * P;
    u32x4 xr[UNITS];
    uint32_t xs[MX ? UNITS : 1];
    auto fetch = [&](int n0, int s) {
        const int rows = a.B - n0 < R ? a.B - n0 : R;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int at = lane + 64 * j, r = at / ROW_UNITS, u = at & (ROW_UNITS - 1);
            const int k = (step0 + s) * W4_STEP + (MX ? 16 : 8) * u;
            xr[j] = u32x4{0, 0, 0, 0};
            if constexpr (MX) xs[j] = 0;
            if (r < rows && k < a.D) {
                const int64_t row = n0 + r;
                xr[j] = *reinterpret_cast<const u32x4*>(a.X + row * a.ldx + (MX ? k : 2 * k));
                if constexpr (MX) xs[j] = a.xs[row * a.ldxs + (k >> 5)];
            }
        }
    };
    auto stage = [&](int rows) {
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int at = lane + 64 * j, r = at / ROW_UNITS, u = at & (ROW_UNITS - 1);
            if (r >= rows) continue;
            if constexpr (MX) {
                const float f = scale_of(xs[j], 0);
                u32x4* to = reinterpret_cast<u32x4*>(mine + ((u >> 1) & 3) * plane + r * (64 * P + 16) + (u >> 3) * 64 + (u & 1) * 32);
                to[0] = w4_features(xr[j][0], xr[j][1], f);
                to[1] = w4_features(xr[j][2], xr[j][3], f);
            } else {
                *reinterpret_cast<u32x4*>(mine + ((u >> 2) & 3) * plane + r * (64 * P + 16) + (u >> 4) * 64 + (u & 3) * 16) = xr[j];
            }
        }
    };
    const int steps = (a.D + W4_STEP - 1) / W4_STEP;
    const bool busy = step0 < steps;                                               // waves beyond the contraction only add up
    if (busy) fetch(row0, 0);                                                         // from the cache, and staged while the codes are on their way
    W4Piece<S> codes[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) w4_load(codes[c], W4Tile(a, busy ? first + 16 * c : a.C), l, step0 * W4_STEP);
    for (int n0 = row0; n0 < a.B; n0 += stride) {
        const int rows = a.B - n0 < R ? a.B - n0 : R;
        f32x4 acc[CT][NT];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[c][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (busy) {
            uint32_t joined[CT][W4Piece<S>::HELD];
            const char* x[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n] = mine + g * plane + (16 * n + i16 < rows ? 16 * n + i16 : rows - 1) * (64 * P + 16);
#pragma unroll
            for (int s0 = 0; s0 < S; s0 += P) {
                stage(rows);
                if (s0 + P < S) {
                    fetch(n0, s0 + P);
                } else if (n0 + stride < a.B) {
                    fetch(n0 + stride, 0);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");             // LDS serves a wave's accesses in their order
                if (s0 == 0)
#pragma unroll
                    for (int c = 0; c < CT; ++c) w4_join(joined[c], codes[c]);
#pragma unroll
                for (int s = s0; s < s0 + P; ++s) {
                    if (step0 + s >= steps) continue;
                    float f[CT];
                    u32x4 v[CT];
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        f[c] = w4_scale<false>(joined[c], s, a.D - step0 * W4_STEP, l);
                        v[c] = w4_codes(codes[c], s, l);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16x8 xb[NT];
#pragma unroll
                        for (int n = 0; n < NT; ++n) xb[n] = *reinterpret_cast<const bf16x8*>(x[n] + 64 * (s - s0) + 16 * q);
#pragma unroll
                        for (int c = 0; c < CT; ++c) {
                            const bf16x8 wa = w4_values(v[c][q], f[c]);
#pragma unroll
                            for (int n = 0; n < NT; ++n) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, xb[n], acc[c][n], 0, 0, 0);
                        }
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (16 * n + i16 < rows) {
                float* to = reinterpret_cast<float*>(mine) + (16 * n + i16) * PITCH + 4 * g;
#pragma unroll
                for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4*>(to + 16 * c) = acc[c][n];
            }
        wait_counts<NO_VM_WAIT, 0>();
        raw_barrier();                                                             // loads stay in flight
        const char* from = lds + 16 * c4;
        for (int r = tid / QUADS; r < rows; r += W4_FEW_THREADS / QUADS) {
            f32x4 z = *reinterpret_cast<const f32x4*>(from + r * PITCH * 4);
            for (int k = 1; k < W4_FEW_WAVES; ++k) z += *reinterpret_cast<const f32x4*>(from + k * region + r * PITCH * 4);
            z += bias;
            if constexpr (TOP1) {
                float best = -INFINITY;
                int at = INT_MAX;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (cls + e < a.C) better_of(best, at, z[e], cls + e);
                for (int m = 1; m < QUADS; m <<= 1) better_of(best, at, __shfl_xor(best, m, 64), __shfl_xor(at, m, 64));       // a row's lanes are neighbours
                if (c4 == 0) {
                    a.part_val[(int64_t)(n0 + r) * gridDim.x + blockIdx.x] = best;
                    a.part_cls[(int64_t)(n0 + r) * gridDim.x + blockIdx.x] = at;
                }
            } else {
                w4_store(a.Z + (int64_t)(n0 + r) * a.ldz + cls, z, a.C - cls);
            }
        }
        if (n0 + stride < a.B) {
            wait_counts<NO_VM_WAIT, 0>();
            raw_barrier();                                                         // the sums have been read
        }
    }
}

// The arg-max's candidates of a row, `parts` of them, shard-local classes, one workgroup to a row.  Any logit that compares, -infinity too, leaves a
// candidate with a class; a row without one has nothing but NaNs, and reports that with the shard's first class.
__global__ __launch_bounds__(256) void w4_merge_top1(const float* __restrict__ val, const int* __restrict__ cls, int parts, int class_offset,
                                                     float* __restrict__ top_logit, int* __restrict__ top_class) {
    __shared__ float sv[4];
    __shared__ int sc[4];
    const int64_t row = (int64_t)blockIdx.x * parts;
    float best = -INFINITY;
    int at = INT_MAX;
    for (int p = threadIdx.x; p < parts; p += 256) better_of(best, at, val[row + p], cls[row + p]);
    for (int m = 32; m > 0; m >>= 1) better_of(best, at, __shfl_xor(best, m, 64), __shfl_xor(at, m, 64));
    if ((threadIdx.x & 63) == 0) {
        sv[threadIdx.x >> 6] = best;
        sc[threadIdx.x >> 6] = at;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) better_of(best, at, sv[w], sc[w]);
        const bool compares = at != INT_MAX;
        top_logit[blockIdx.x] = compares ? best : __uint_as_float(0x7fc00000u);
        top_class[blockIdx.x] = compares ? at + class_offset : class_offset;
    }
}

static inline bool al(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int S, int CT, int NT, bool MX, bool TOP1>
static void launch_w4_few(const W4Args& a, const W4Plan& f, hipStream_t s) {
    const size_t bytes = (size_t)W4_FEW_WAVES * w4_few_region(w4_few_piece(S, CT, NT, MX), CT, a.B < 16 * NT ? a.B : 16 * NT);
    hipLaunchKernelGGL((w4_few<S, CT, NT, MX, TOP1>), dim3(f.groups, f.row_groups), dim3(W4_FEW_THREADS), bytes, s, a);
}

template <int NT, bool MX, bool TOP1>
static void launch_w4_steps(const W4Args& a, const W4Plan& f, hipStream_t s) {
    switch (f.S * 8 + f.CT) {
        case 1 * 8 + 4: return launch_w4_few<1, 4, NT, MX, TOP1>(a, f, s);
        case 2 * 8 + 1: return launch_w4_few<2, 1, NT, MX, TOP1>(a, f, s);
        case 2 * 8 + 4: return launch_w4_few<2, 4, NT, MX, TOP1>(a, f, s);
        case 4 * 8 + 1: return launch_w4_few<4, 1, NT, MX, TOP1>(a, f, s);
        case 4 * 8 + 2: return launch_w4_few<4, 2, NT, MX, TOP1>(a, f, s);
        default: return launch_w4_few<8, 1, NT, MX, TOP1>(a, f, s);
    }
}

template <int NT, int CT, int WAVES, bool MX, bool TOP1>
static void launch_w4_tiles(const W4Args& a, const W4Plan& p, hipStream_t s) {
    const int row_blocks = (a.B + 16 * NT - 1) / (16 * NT), parts = TOP1 ? w4_parts(p, a.B) : p.groups;
    const int64_t blocks = ((int64_t)parts + 7) / 8 * 8 * row_blocks;
    hipLaunchKernelGGL((w4_tiles<NT, CT, WAVES, MX, TOP1>), dim3((unsigned)blocks), dim3(64 * WAVES), 0, s, a, p.groups, row_blocks, parts);
}

template <int NT, int RING, bool MX, bool TOP1>
static void launch_w4_stream(const W4Args& a, const W4Plan& p, hipStream_t s) {
    size_t bytes = w4_stream_lds(a.B, a.D);
    const size_t least = TOP1 ? (size_t)W4_STREAM_WAVES * 16 * NT * 8 : 0;
    if (bytes < least) bytes = least;
    hipLaunchKernelGGL((w4_stream<NT, RING, MX, TOP1>), dim3(p.groups), dim3(W4_STREAM_THREADS), bytes, s, a, (int)(((int64_t)a.C + 15) / 16));
}

template <bool MX, bool TOP1>
static void launch_w4_type(const W4Args& a, hipStream_t s) {
    const W4Plan p = w4_plan(a.B, a.D, a.C, TOP1);
    if (p.way == W4_FEW) return a.B > 16 ? launch_w4_steps<2, MX, TOP1>(a, p, s) : launch_w4_steps<1, MX, TOP1>(a, p, s);
    if (p.way == W4_STREAM) {
        if (a.B > 16) return launch_w4_stream<2, 1, MX, TOP1>(a, p, s);
        return p.ring == 1 ? launch_w4_stream<1, 1, MX, TOP1>(a, p, s) : launch_w4_stream<1, 2, MX, TOP1>(a, p, s);
    }
    if (!p.wide) return p.NT == 2 ? launch_w4_tiles<2, 2, 4, MX, TOP1>(a, p, s) : launch_w4_tiles<4, 2, 4, MX, TOP1>(a, p, s);
    switch (p.NT) {
        case 2: return launch_w4_tiles<2, 2, 8, MX, TOP1>(a, p, s);
        case 4: return launch_w4_tiles<4, 2, 8, MX, TOP1>(a, p, s);
        default: break;
    }
    if constexpr (!TOP1)
        switch (p.NT) {
            case 5: return launch_w4_tiles<5, 4, 8, MX, false>(a, p, s);
            case 6: return launch_w4_tiles<6, 4, 8, MX, false>(a, p, s);
            case 7: return launch_w4_tiles<7, 4, 8, MX, false>(a, p, s);
            default: return launch_w4_tiles<8, 4, 8, MX, false>(a, p, s);
        }
}

template <bool TOP1>
static void launch_w4(const W4Args& a, hipStream_t s) {
    if (a.xs != nullptr) launch_w4_type<true, TOP1>(a, s);
    else launch_w4_type<false, TOP1>(a, s);
}

static int check_w4(const void* X, int64_t ldx, const void* X_scales, int64_t ldxs, const void* W4, int64_t ldw4, const void* W_scales,
                    int64_t lds, const float* b_shard, int32_t B, int32_t D, int32_t C_shard) {
    if (!X || !W4 || !W_scales) return WS_ERR_NULL;
    if (B <= 0 || D <= 0 || C_shard <= 0 || D % 64 || B > W4_MAX_ROWS) return WS_ERR_SHAPE;
    if (ldw4 > W4_MAX_PITCH || lds > W4_MAX_PITCH) return WS_ERR_SHAPE;
    if (C_shard > W4_MAX_CLASSES) return WS_ERR_RANGE;
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

// Whatever the number of features.
size_t ws_w4_top1_workspace_bytes(int32_t B, int32_t C_shard) {
    if (B <= 0 || C_shard <= 0 || B > W4_MAX_ROWS) return 0;
    return (size_t)w4_most_parts(B, C_shard) * B * 8;
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
    const int parts = w4_parts(w4_plan(B, D, C_shard, true), B);
    a.part_val = static_cast<float*>(workspace);
    a.part_cls = reinterpret_cast<int*>(a.part_val + (int64_t)parts * B);
    hipStream_t s = static_cast<hipStream_t>(stream);
    launch_w4<true>(a, s);
    hipLaunchKernelGGL(w4_merge_top1, dim3(B), dim3(256), 0, s, a.part_val, a.part_cls, parts, class_offset, top_logit, top_class);
    return hipGetLastError() == hipSuccess ? WS_OK : WS_ERR_HIP;
}

}  // extern "C"
