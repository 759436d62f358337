// Operands of the 8-bit products: e4m3 values with a scale for each block of 128 channels of one row (activations) or of 128 rows (weights),
//   scale = the smallest power of two with amax <= 448 scale,   q = e4m3(x / scale)   (nearest, ties to even).
// With a power of two the division is exact, so that every q is the nearest e4m3 value to x / scale, whatever x is; a scale of amax / 448 has no smaller
// relative error (e4m3 values are 2^-4 apart wherever they lie), and rounds x / scale once more, to the wrong side of a border wherever bf16 inputs
// put x / scale on one.  amax counts as 2^-100 at least.  A block with an infinity or a NaN has the scale NaN and values NaN.
//
// Bound by memory: 2 or 4 bytes read and 1 written per value.  A lane has 16 channels (whole sectors), 8 lanes a block of a row.
// us, bf16: rows of 32760 x 1536 26.0 (0.89 of the copy rate), a weight of 13824 x 5120 33.5 (0.97).
#pragma once
#include "norm.cuh"

namespace carnator {
namespace fp8 {

constexpr int kBlock = 128;              // channels, and rows of a weight's block, that share a scale
constexpr int kLaneChannels = 16, kLanes = kBlock / kLaneChannels;

// The bits of the largest magnitude -> scale and its reciprocal.  448 = 1.75 x 2^8.
__device__ __forceinline__ void scale_of(uint32_t amax_bits, float& scale, float& inverse) {
    const uint32_t least = (127u - 100u) << 23, b = amax_bits < least ? least : amax_bits;
    const uint32_t e = (b >> 23) - 8u + ((b & 0x7FFFFFu) > 0x600000u ? 1u : 0u);
    scale = __uint_as_float(e << 23);
    inverse = __uint_as_float((254u - e) << 23);
    if (b >= 0x7F800000u) scale = inverse = __uint_as_float(0x7FC00000u);
}
// two values -> two e4m3 in the low 16 bits
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// 16 channels of a row, of which n are there (none: zeros)
template <bool F32>
struct Lane16 {
    static constexpr int kWords = F32 ? 16 : 8;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* base, int64_t off, int n) {
        const char* p = static_cast<const char*>(base) + off * (F32 ? 4 : 2);
        if (n >= kLaneChannels) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "l"(p + 16 * i));
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = 0;
            if (n <= 0) return;
#pragma unroll
            for (int i = 0; i < kLaneChannels; ++i)
                if (i < n) {
                    if (F32) w[F32 ? i : 0] = reinterpret_cast<const volatile uint32_t*>(p)[i];
                    else w[F32 ? 0 : i / 2] |= uint32_t(reinterpret_cast<const volatile uint16_t*>(p)[i]) << (16 * (i & 1));
                }
        }
    }
    // bits of the largest magnitude: those of a NaN are above all others
    __device__ __forceinline__ uint32_t most() const {
        if (F32) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kWords; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
            return m;
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7FFF7FFFu));
        return max(m << 16, m & 0xFFFF0000u);
    }
    __device__ __forceinline__ float get(int i) const {
        if (F32) return __uint_as_float(w[F32 ? i : 0]);
        return __uint_as_float(i & 1 ? w[F32 ? 0 : i / 2] & 0xFFFF0000u : w[F32 ? 0 : i / 2] << 16);
    }
    __device__ __forceinline__ uint4 quantized(float inverse) const {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = e4m3x2(get(4 * i) * inverse, get(4 * i + 1) * inverse) | e4m3x2(get(4 * i + 2) * inverse, get(4 * i + 3) * inverse) << 16;
        return make_uint4(q[0], q[1], q[2], q[3]);
    }
};
__device__ __forceinline__ void store_q(uint8_t* p, const uint4& q, int n) {
    if (n >= kLaneChannels) {
        *reinterpret_cast<uint4*>(p) = q;
    } else {
        const uint32_t t[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < kLaneChannels; ++i) if (i < n) p[i] = uint8_t(t[i / 4] >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ uint32_t block_most(uint32_t m) {       // over the 8 lanes of a block
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
}

struct QuantArgs {
    const void* x; uint8_t* q; float* scale;
    int64_t xs[2], qs[2];                // (batch, row)
    int64_t ss[3];                       // (batch, row or block of rows, block)
    int batches, rows, cols, blocks;
};

// A scale per row: 8 lanes a block, kAhead blocks of a row on their way per lane.  The groups of 8 lanes of `ctas` CTAs walk over (row, run of kAhead blocks);
// put(row, block, scales) is called by one lane of each, with those of kAhead blocks (past the last block: of zeros).
constexpr int kRowThreads = 256;
template <bool F32> constexpr int kAheadOf = F32 ? 2 : 4;
template <bool F32, int kAhead, typename Put>
__device__ __forceinline__ void quantize_rows(const QuantArgs& a, int b, int cta, int ctas, Put put) {
    const int l = threadIdx.x % kLanes, runs = (a.blocks + kAhead - 1) / kAhead;
    const int64_t items = int64_t(a.rows) * runs, step = int64_t(ctas) * (kRowThreads / kLanes);
    // warp-uniform trips: the lanes of a warp exchange their largest values
    for (int64_t first = int64_t(cta) * (kRowThreads / kLanes) + threadIdx.x / 32 * (32 / kLanes); first < items; first += step) {
        const int64_t item = first + threadIdx.x % 32 / kLanes;
        const bool on = item < items;
        const int row = on ? int(item / runs) : 0, blk = on ? int(item - int64_t(row) * runs) * kAhead : 0;
        Lane16<F32> v[kAhead];
        int n[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int col = (blk + k) * kBlock + l * kLaneChannels;
            n[k] = on ? min(max(a.cols - col, 0), kLaneChannels) : 0;
            v[k].load(a.x, b * a.xs[0] + row * a.xs[1] + col, n[k]);
        }
        float scale[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float inverse;
            scale_of(block_most(v[k].most()), scale[k], inverse);
            if (n[k] > 0) store_q(a.q + b * a.qs[0] + row * a.qs[1] + (blk + k) * kBlock + l * kLaneChannels, v[k].quantized(inverse), n[k]);
        }
        if (on && l == 0) put(row, blk, scale);
    }
}
template <bool F32, int kAhead>
__global__ void __launch_bounds__(kRowThreads, 4) quantize_rows_kernel(const QuantArgs a) {
    const int b = blockIdx.y;
    grid_launch_dependents();
    grid_wait();
    quantize_rows<F32, kAhead>(a, b, blockIdx.x, gridDim.x, [&](int row, int blk, const float (&scale)[kAhead]) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (blk + k < a.blocks) a.scale[b * a.ss[0] + row * a.ss[1] + (blk + k) * a.ss[2]] = scale[k];
    });
}

// A scale per 128 x 128: a CTA per block, four rows per lane.
constexpr int kTileThreads = 256;
template <bool F32>
__global__ void __launch_bounds__(kTileThreads) quantize_tiles_kernel(const QuantArgs a) {
    __shared__ uint32_t part[kTileThreads / 32];
    const int l = threadIdx.x % kLanes, g = threadIdx.x / kLanes, b = blockIdx.y;
    const int tile = blockIdx.x / a.blocks, blk = blockIdx.x - tile * a.blocks;
    const int col = blk * kBlock + l * kLaneChannels;
    constexpr int kRows = kBlock / (kTileThreads / kLanes);
    grid_launch_dependents();
    grid_wait();
    Lane16<F32> v[kRows];
    int n[kRows];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const int row = tile * kBlock + g + k * (kTileThreads / kLanes);
        n[k] = row < a.rows ? min(max(a.cols - col, 0), kLaneChannels) : 0;
        v[k].load(a.x, b * a.xs[0] + row * a.xs[1] + col, n[k]);
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) m = max(m, v[k].most());
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileThreads / 32; ++w) m = max(m, part[w]);
    float scale, inverse;
    scale_of(m, scale, inverse);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const int row = tile * kBlock + g + k * (kTileThreads / kLanes);
        if (n[k] > 0) store_q(a.q + b * a.qs[0] + row * a.qs[1] + col, v[k].quantized(inverse), n[k]);
    }
    if (threadIdx.x == 0) a.scale[b * a.ss[0] + tile * a.ss[1] + blk * a.ss[2]] = scale;
}

// ---- host side ------------------------------------------------------------------------------------
// CTAs of a run each; the walk is for what passes a grid's size.  (Four CTAs an SM that walk over 2.6 runs each: 32760 x 1536 26.3 us.)
inline int row_ctas(const QuantArgs& a, bool f32) {
    const int64_t items = int64_t(a.rows) * ceil_div(a.blocks, f32 ? kAheadOf<true> : kAheadOf<false>), ctas = (items + kRowThreads / kLanes - 1) / (kRowThreads / kLanes);
    return int(std::min<int64_t>(ctas, 1 << 24));
}
inline cudaError_t launch_quantize(const QuantArgs& a, bool f32, int block_rows, cudaStream_t stream) {
    if (block_rows == 1) {
        const dim3 grid(unsigned(row_ctas(a, f32)), unsigned(a.batches));
        return f32 ? launch_dependent(quantize_rows_kernel<true, kAheadOf<true>>, grid, dim3(kRowThreads), 0, stream, a)
                   : launch_dependent(quantize_rows_kernel<false, kAheadOf<false>>, grid, dim3(kRowThreads), 0, stream, a);
    }
    const dim3 grid(unsigned(ceil_div(a.rows, kBlock) * a.blocks), unsigned(a.batches));
    return f32 ? launch_dependent(quantize_tiles_kernel<true>, grid, dim3(kTileThreads), 0, stream, a)
               : launch_dependent(quantize_tiles_kernel<false>, grid, dim3(kTileThreads), 0, stream, a);
}

}  // namespace fp8
}  // namespace carnator
