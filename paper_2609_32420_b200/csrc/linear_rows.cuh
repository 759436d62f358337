// The projection's product for a few rows (the conditioning of a denoising step: one row per batch entry):
//   z = x W^T + bias,   y = residual + gate_b act(z),   up to 16 rows.
// All it has to move is W, once.  A CTA takes 16 rows of W (output features); its warps share k, and a lane fetches W straight
// into the registers of the matrix instruction: mma.m16n8k16 wants k = 2t, 2t+1, 2t+8, 2t+9 from lane t of a quad, but a sum over k may be taken
// in any order, so lane t reads 8 consecutive k (16 bytes) of its row and gives them to two instructions, and the x operand is read the same way.
// No shared memory and no barrier until the warps' partial sums are added, in the order of k.
#pragma once
#include "linear_tcgen05.cuh"

namespace carnator {
namespace lin {

// Rows of x per call that this kernel takes: one column tile of the instruction, or two where W is not large (16 rows of 1536 x 1536: 4.0 us, on tcgen05
// 10.2; of 1536 x 9216 6.9 and 14.2; of 8960 x 1536 12.3 and 13.4; but of 5120 x 30720, whose x every CTA reads again, 78.9 and 63.3).
constexpr int kRowsMost = 16, kRowsOneTile = 8;
constexpr int64_t kRowsWeights = int64_t(1) << 26;
inline bool rows_take(int64_t rows, int64_t in_features, int64_t out_features) {
    return rows <= kRowsOneTile || (rows <= kRowsMost && in_features * out_features < kRowsWeights);
}

struct RowsArgs {
    Epilogue e;
    const __nv_bfloat16* x; const __nv_bfloat16* w;
    int64_t xs[2], w_stride;
    WsHeader* hdr;
    int rows, per_batch, K, cols;        // rows over all batch entries; rows of an entry
};

__device__ __forceinline__ uint4 load_k8(const __nv_bfloat16* row, int k, int K) {
    if (k + 8 <= K) {                    // not through the read-only path: the kernel ahead may write it while this one is resident
        uint4 v;
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + k));
        return v;
    }
    uint32_t t[4] = {0, 0, 0, 0};        // the last k of a row: what lies behind them is not the row's
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K) t[i / 2] |= uint32_t(reinterpret_cast<const uint16_t*>(row)[k + i]) << (16 * (i & 1));
    return make_uint4(t[0], t[1], t[2], t[3]);
}
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT: column tiles of 8 rows of x; kRowsWarps: warps that share k; kRuns: a warp's sums are longer than kLongRun (a loop around the loop, which takes
// registers and with them one CTA in seven: 2 x 5120 x 30720 76.7 us with it, 69.6 without, cold caches and launch included).
template <int NT, int kRowsWarps, bool kRuns>
__global__ void __launch_bounds__(32 * kRowsWarps) linear_rows_kernel(const RowsArgs a) {
    __shared__ float sums[kRowsWarps][16][8 * NT + 1];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    grid_launch_dependents();
    grid_wait();                         // launched while the kernel ahead drains
    if (blockIdx.x == 0 && tid == 0) a.hdr->status = 0;
    const int f0 = blockIdx.x * 16;
    const bool on0 = f0 + g < a.cols, on1 = f0 + g + 8 < a.cols;
    const __nv_bfloat16* w0 = a.w + int64_t(f0 + g) * a.w_stride;
    const __nv_bfloat16* w1 = w0 + 8 * a.w_stride;
    const __nv_bfloat16* xr[NT];
    bool xon[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int row = j * 8 + g;
        xon[j] = row < a.rows;
        const int b = xon[j] ? row / a.per_batch : 0;
        xr[j] = a.x + b * a.xs[0] + (xon[j] ? row - b * a.per_batch : 0) * a.xs[1];
    }
    // Two sums per warp, emptied into shared memory after every kLongRun of k: the instruction cuts its sums off, and what that loses grows with their length
    // (1 x 65536 x 7200 onto fp32, four warps: error 9.0e-6 in one run).
    float d[NT][4], d2[NT][4];
    const uint4 zero = make_uint4(0, 0, 0, 0);
    constexpr int U = 4;                 // pieces of 32 k in flight per warp
    const int pieces = (a.K + 31) / 32;
    int p = warp;
    do {
        const bool first = !kRuns || p == warp;
        const int stop = kRuns ? min(pieces, p + kRowsWarps * (kLongRun / 16)) : pieces;        // a piece gives each sum 16 k
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) { d[j][i] = 0.f; d2[j][i] = 0.f; }
        for (; p < stop; p += kRowsWarps * U) {
            uint4 u0[U], u1[U], xv[U][NT];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int k = (p + q * kRowsWarps) * 32 + t * 8;         // past the end: zero
                u0[q] = on0 ? load_k8(w0, k, a.K) : zero;
                u1[q] = on1 ? load_k8(w1, k, a.K) : zero;
#pragma unroll
                for (int j = 0; j < NT; ++j) xv[q][j] = xon[j] ? load_k8(xr[j], k, a.K) : zero;
            }
#pragma unroll
            for (int q = 0; q < U; ++q)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma_16x8x16(d[j], u0[q].x, u1[q].x, u0[q].y, u1[q].y, xv[q][j].x, xv[q][j].y);
                    mma_16x8x16(d2[j], u0[q].z, u1[q].z, u0[q].w, u1[q].w, xv[q][j].z, xv[q][j].w);
                }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)     // d0, d1: feature g, rows 2t and 2t + 1 of x; d2, d3: feature g + 8
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float& at = sums[warp][g + 8 * (i >> 1)][j * 8 + 2 * t + (i & 1)];
                at = first ? d[j][i] + d2[j][i] : at + (d[j][i] + d2[j][i]);
            }
    } while (kRuns && p < pieces);
    __syncthreads();
    auto param = [&](const void* p, int64_t i, int f32) { return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); };
    const int f = tid & 15, col = f0 + f;
    for (int row = tid >> 4; row < a.rows && col < a.cols; row += 2 * kRowsWarps) {
        float z = 0.f;
#pragma unroll
        for (int k = 0; k < kRowsWarps; ++k) z += sums[k][f][row];
        const int b = row / a.per_batch, r = row - b * a.per_batch;
        if (a.e.bias) z += param(a.e.bias, col, a.e.bias_f32);
        if (a.e.z) static_cast<__nv_bfloat16*>(a.e.z)[b * a.e.zs[0] + r * a.e.zs[1] + col] = __float2bfloat16_rn(z);
        float y = a.e.act == kActGeluTanh ? activation<kActGeluTanh>(z) : a.e.act == kActGelu ? activation<kActGelu>(z)
                : a.e.act == kActSilu ? activation<kActSilu>(z) : z;
        if (a.e.gate) y *= param(a.e.gate, b * a.e.gate_stride + col, a.e.gate_f32);
        if (a.e.residual) y += param(a.e.residual, b * a.e.rs[0] + r * a.e.rs[1] + col, a.e.y_f32);
        const int64_t off = b * a.e.ys[0] + r * a.e.ys[1] + col;
        if (a.e.y_f32) static_cast<float*>(a.e.y)[off] = y;
        else static_cast<__nv_bfloat16*>(a.e.y)[off] = __float2bfloat16_rn(y);
    }
}

// Warps that share k: many where there are few CTAs, so that all of W is on its way at once (1536 x 1536, 96 CTAs: 16 warps 3.0 us, 8 4.5), few where
// CTAs fill the SMs several times over (30720 x 5120, 1920 CTAs: 4 warps 49.0 us, 8 53.5, 16 82; 5120 x 5120, 320 CTAs: 8 warps 8.7 us, 4 14, 16 15).
static_assert(kRowsWeights <= int64_t(2 * kLongRun * 8) * 16 * 148, "more than 8 rows: fewer than 16 warps share k only where it needs no runs");
template <int NT>
inline cudaError_t launch_rows_tiles(const RowsArgs& a, cudaStream_t stream) {
    const int grid = ceil_div(a.cols, 16);
    const int warps = grid <= 148 ? 16 : grid <= 3 * 148 ? 8 : 4;
    const bool runs = a.K > 2 * kLongRun * warps;        // with two column tiles only where 16 warps share k: W is not large then
    auto kern = warps == 16 ? (runs ? linear_rows_kernel<NT, 16, true> : linear_rows_kernel<NT, 16, false>)
              : warps == 8  ? (runs ? linear_rows_kernel<1, 8, true> : linear_rows_kernel<NT, 8, false>)
                            : (runs ? linear_rows_kernel<1, 4, true> : linear_rows_kernel<NT, 4, false>);
    return launch_dependent(kern, dim3(grid), dim3(32 * warps), 0, stream, a);
}

inline cudaError_t launch_rows(const RowsArgs& a, cudaStream_t stream) {
    return a.rows <= 8 ? launch_rows_tiles<1>(a, stream) : launch_rows_tiles<2>(a, stream);
}

}  // namespace lin
}  // namespace carnator
