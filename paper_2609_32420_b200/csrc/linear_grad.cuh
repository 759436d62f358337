// The elementwise half of a projection's gradients: from dy, the saved pre-activation z and the gate,
//   dz = dy gate_b act'(z),   dbias = sum over rows of dz,   dgate_b = sum over the rows of entry b of dy act(z).
// One pass over dy and z, the rows ahead of a warp on their way into shared memory (from registers, two rows at a time, 32760 x 8960 with GELU took 449 us
// instead of 417, a product of 8 columns included); dz is rounded to bf16 here, because the two products behind it take 16-bit operands (its rounding adds as much error to
// dX and dW as their own does: against 64 bits 2.34e-3 instead of 1.66e-3; in two 16-bit terms it would double the products).  The sums are taken from the unrounded values: a thread keeps 8 columns over every eighth row of
// its CTA's rows, a CTA leaves one partial row, a second kernel adds those in a fixed order.
#pragma once
#include "linear_tcgen05.cuh"

namespace carnator {
namespace lin {

struct GradArgs {
    const void* dy; const __nv_bfloat16* z; const void* gate;
    __nv_bfloat16* dz;                   // [batches, rows, ...] or NULL: only the sums are wanted
    float* part_bias; float* part_gate;  // [batches * chunks][cols] or NULL
    int64_t ds[2], zs[2], dzs[2], gate_stride;
    int act, dy_f32, gate_f32;
    int rows, cols, chunks;              // rows and chunks of rows of a batch entry
};

constexpr int kGradCols = 256, kGradLanes = 8;       // columns and row lanes of a CTA
constexpr int kGradPerSm = 3;                        // CTAs that share an SM
constexpr int kGradStages = 4;                       // rows ahead of each warp

template <int ACT, bool DYF>
__global__ void __launch_bounds__(32 * kGradLanes, kGradPerSm) linear_grad_kernel(const GradArgs a) {
    extern __shared__ uint4 grad_smem[];
    auto sums = reinterpret_cast<float (*)[kGradLanes][kGradCols + 8]>(grad_smem);       // in the place of the rows, when all have been read
    constexpr uint32_t kDyBytes = 32 * kGradLanes * 16 * (DYF ? 2 : 1), kZBytes = 32 * kGradLanes * 16;
    grid_launch_dependents();
    grid_wait();
    const int cv = threadIdx.x & 31, rl = threadIdx.x >> 5, b = blockIdx.z;
    const int col = blockIdx.x * kGradCols + cv * 8, n = min(max(a.cols - col, 0), 8);
    const int r0 = int(int64_t(blockIdx.y) * a.rows / a.chunks), r1 = int(int64_t(blockIdx.y + 1) * a.rows / a.chunks);
    norm::Eight sb, sg, gate;
    {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = 1.f;
        if (a.gate) norm::load_param8(a.gate, b * a.gate_stride + col, a.gate_f32, 0, n, t);
        gate = norm::eight_of(t);
#pragma unroll
        for (int i = 0; i < 4; ++i) { sb.p[i] = two(0.f); sg.p[i] = two(0.f); }
    }
    const uint32_t ring = uint32_t(__cvta_generic_to_shared(grad_smem)), z_at = kDyBytes, stage = kDyBytes + kZBytes;
    const norm::Stage<DYF, 1, 32> in(blockIdx.x * 32 + cv);
    const norm::Stage<false, 1, 32> in_z(blockIdx.x * 32 + cv);
    const char* dy = static_cast<const char*>(a.dy) + (b * a.ds[0] + in.col) * (DYF ? 4 : 2);
    const char* zp = reinterpret_cast<const char*>(a.z) + (b * a.zs[0] + in_z.col) * 2;
    int ahead = r0 + rl;
    auto fetch = [&](int s) {
        const bool on = ahead < r1;
        in.copy(ring + uint32_t(s) * stage, dy + ahead * a.ds[1] * (DYF ? 4 : 2), (a.cols - in.col) * (DYF ? 4 : 2), 0, on);
        if (a.z) in_z.copy(ring + uint32_t(s) * stage + z_at, zp + ahead * a.zs[1] * 2, (a.cols - in_z.col) * 2, 0, on);
        norm::copies_commit();
        ahead += kGradLanes;
    };
#pragma unroll
    for (int s = 0; s < kGradStages; ++s) fetch(s);
    int s = 0;
    for (int row = r0 + rl; row < r1; row += kGradLanes) {
        norm::copies_wait(kGradStages - 1);
        if (DYF) __syncwarp();
        norm::Eight d = in.read(ring + uint32_t(s) * stage, 0), z;
        if (a.z) z = in_z.read(ring + uint32_t(s) * stage + z_at, 0);
        if (DYF) __syncwarp();
        fetch(s);                        // into the place just read
        if (++s == kGradStages) s = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f2 f = two(0.f), k = two(1.f);
            if (a.z) act_and_slope<ACT>(z.p[i], f, k);
            if (a.part_gate) sg.p[i] = fma2(d.p[i], f, sg.p[i]);
            if (a.gate) d.p[i] = mul2(d.p[i], gate.p[i]);
            if (ACT != kActNone) d.p[i] = mul2(d.p[i], k);
            sb.p[i] = add2(sb.p[i], d.p[i]);
        }
        if (a.dz) norm::store_eight<false>(a.dz, b * a.dzs[0] + row * a.dzs[1] + col, d, n, false);
    }
    norm::copies_wait(0);
    if (!a.part_bias && !a.part_gate) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        one_each(sb.p[i], sums[0][rl][cv * 8 + 2 * i], sums[0][rl][cv * 8 + 2 * i + 1]);
        one_each(sg.p[i], sums[1][rl][cv * 8 + 2 * i], sums[1][rl][cv * 8 + 2 * i + 1]);
    }
    __syncthreads();
    const int c = blockIdx.x * kGradCols + threadIdx.x;
    if (c >= a.cols) return;
    float tb = 0.f, tg = 0.f;
#pragma unroll
    for (int k = 0; k < kGradLanes; ++k) { tb += sums[0][k][threadIdx.x]; tg += sums[1][k][threadIdx.x]; }
    const int64_t out = (int64_t(b) * a.chunks + blockIdx.y) * a.cols + c;
    if (a.part_bias) a.part_bias[out] = tb;
    if (a.part_gate) a.part_gate[out] = tg;
}

// dbias = sum over all partial rows, dgate of an entry over its own: 32 columns per CTA, as norm_reduce_kernel
struct GradReduceArgs { const float* part_bias; const float* part_gate; float* dbias; float* dgate; int batches, chunks, cols; };
constexpr int kGradReduceWarps = 16;
__global__ void __launch_bounds__(32 * kGradReduceWarps) linear_grad_reduce_kernel(const GradReduceArgs a) {
    __shared__ float sums[2][kGradReduceWarps][32];
    grid_launch_dependents();
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float total = 0.f;
    for (int b = 0; b < a.batches; ++b) {
        float p = 0.f, g = 0.f;
        if (c < a.cols)
#pragma unroll 4
            for (int k = warp; k < a.chunks; k += kGradReduceWarps) {
                const int64_t at = (int64_t(b) * a.chunks + k) * a.cols + c;
                if (a.dbias) p += a.part_bias[at];
                if (a.dgate) g += a.part_gate[at];
            }
        sums[0][warp][lane] = p;
        sums[1][warp][lane] = g;
        __syncthreads();
        if (warp == 0 && c < a.cols) {
            p = 0.f; g = 0.f;
#pragma unroll
            for (int k = 0; k < kGradReduceWarps; ++k) { p += sums[0][k][lane]; g += sums[1][k][lane]; }
            total += p;
            if (a.dgate) a.dgate[int64_t(b) * a.cols + c] = g;
        }
        __syncthreads();
    }
    if (warp == 0 && c < a.cols && a.dbias) a.dbias[c] = total;
}

// Chunks of rows per batch entry: one wave of CTAs over the columns, none with fewer than 32 rows.
inline int grad_chunks(int64_t batches, int64_t rows, int64_t cols) {
    const int64_t strips = (cols + kGradCols - 1) / kGradCols, want = 148 * kGradPerSm / (strips * batches);
    return int(std::max<int64_t>(1, std::min(want, rows / 32)));
}

template <int ACT>
inline cudaError_t launch_grad_act(const GradArgs& a, dim3 grid, cudaStream_t stream) {
    const size_t stage = size_t(32) * kGradLanes * 16 * (a.dy_f32 ? 3 : 2);          // dy and z: 48 KB at most, no need to ask for more
    return launch_dependent(a.dy_f32 ? linear_grad_kernel<ACT, true> : linear_grad_kernel<ACT, false>, grid, dim3(32 * kGradLanes), kGradStages * stage, stream, a);
}
inline cudaError_t launch_grad(const GradArgs& a, int batches, cudaStream_t stream) {
    const dim3 grid(ceil_div(a.cols, kGradCols), a.chunks, batches);
    switch (a.act) {
        case kActGeluTanh: return launch_grad_act<kActGeluTanh>(a, grid, stream);
        case kActGelu: return launch_grad_act<kActGelu>(a, grid, stream);
        case kActSilu: return launch_grad_act<kActSilu>(a, grid, stream);
        default: return launch_grad_act<kActNone>(a, grid, stream);
    }
}

}  // namespace lin
}  // namespace carnator
