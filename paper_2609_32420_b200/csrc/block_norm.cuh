// The end of a block and the beginning of the next one: the block's output x is normed (or not), gated and added to the residual stream r, and the sum is normed and
// modulated for the next block; and its gradients.
//   xh = (x - mu1) rstd1,  p = xh w1 + b1,  s = alpha r + gate_b p,  sh = (s - mu2) rstd2,  y = (sh w2 + b2)(1 + scale_b) + shift_b
// with mu = mean and rstd = (variance + eps)^-1/2 for a layer norm, mu = 0 and rstd = (mean square + eps)^-1/2 for an RMS norm, 0 and 1 for none (the first only).
// Backward, with t = dy w2 (1 + scale_b), and bars for means over the channels (the mean of t itself only for a layer norm):
//   G = ds + rstd2 (t - mean(t) - sh mean(t sh)),   dr = alpha G,   q = G gate_b w1,   dx = rstd1 (q - mean(q) - xh mean(q xh))
//   P1 = sum G xh, S1 = sum G, P2 = sum dy sh, S2 = sum dy over the rows of entry b:
//   dw1 = sum_b gate_b P1, db1 = sum_b gate_b S1, dgate_b = w1 P1 + b1 S1, dw2 = sum_b (1 + scale_b) P2, db2 = .. S2, dscale_b = w2 P2 + b2 S2, dshift_b = S2
//
// Bound by memory: r and x read once, s and y written once (apart, the norms and the sum move x and s three times each).  Rows are worked on as in norm.cuh, whose
// pieces these are: a row's warps copy it into shared memory ahead of time and hold it in registers, 8 channels per lane and access; the sum s stays there between the two
// norms.  Two barriers of the row's warps per row and norm at most.  Sums per channel stay in registers over all rows of a CTA, partial rows are added in a fixed
// order by a second kernel: no atomics, the same bits every time.
#pragma once
#include "norm.cuh"

namespace carnator {
namespace blk {
using namespace norm;

constexpr int kMostChannels = 8192;      // the backward kernel's four sums per channel: 16 channels a lane are what registers hold, of 512 lanes
enum { kNone = 0, kLayer = 1, kRms = 2 };
constexpr int kWarps = 16, kThreads = 32 * kWarps;

struct Args2 {
    const void* r; const void* x; void* s; void* y;       // backward: s is the saved sum, r is ds (or NULL)
    const void* dy; void* dr; void* dx;
    const void* w1; const void* b1; const void* gate;      // [C], [C], [B,C] or NULL
    const void* w2; const void* b2; const void* shift; const void* scale;
    float* stats;                        // [4][B][N]: mean and rstd of either norm, or NULL
    float* part;                         // backward: [B * chunks][4][C] partial P1, S1, P2, S2, or NULL
    int64_t rs[2], xs[2], ss[2], ys[2], dys[2], drs[2], dxs[2];   // element strides of (batch, row)
    int64_t gate_stride, shift_stride, scale_stride;
    int B, N, C, chunks, stages, warps;
    int post, pre, w_f32, mod_f32, vec_ok;
    int wide_s, wide_y, wide_dx;         // rows of the outputs start on 32-byte boundaries
    float alpha, eps1, eps2, inv_c;
};

// gate w1 and gate b1 of 8 channels
__device__ __forceinline__ void factors1(const Args2& a, int b, int col, int n, float (&ka)[8], float (&kc)[8], bool offsets) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { ka[i] = 1.f; kc[i] = 0.f; }
    if (a.w1) load_param8(a.w1, col, a.w_f32, a.vec_ok, n, ka);
    if (offsets && a.b1) load_param8(a.b1, col, a.w_f32, a.vec_ok, n, kc);
    if (a.gate) {
        load_param8(a.gate, b * a.gate_stride + col, a.mod_f32, a.vec_ok, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) { ka[i] *= t[i]; kc[i] *= t[i]; }
    }
}
// w2 (1 + scale) and b2 (1 + scale) + shift
__device__ __forceinline__ void factors2(const Args2& a, int b, int col, int n, float (&ka)[8], float (&kc)[8], bool offsets) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { ka[i] = 1.f; kc[i] = 0.f; }
    if (a.w2) load_param8(a.w2, col, a.w_f32, a.vec_ok, n, ka);
    if (offsets && a.b2) load_param8(a.b2, col, a.w_f32, a.vec_ok, n, kc);
    if (a.scale) {
        load_param8(a.scale, b * a.scale_stride + col, a.mod_f32, a.vec_ok, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) { ka[i] = fmaf(ka[i], t[i], ka[i]); kc[i] = fmaf(kc[i], t[i], kc[i]); }
    }
    if (offsets && a.shift) {
        load_param8(a.shift, b * a.shift_stride + col, a.mod_f32, a.vec_ok, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) kc[i] += t[i];
    }
}

// Mean and squared deviations (layer norm) or sum of squares (RMS) of a row held by a slot's warps; `room`: a float4 per warp of the slot, free until the slot's next
// barrier but one.  As in norm.cuh: deviations around the mean of a warp's own channels, put together by (mean, sum of squares).
template <int V>
__device__ __forceinline__ void moments(const Eight (&f)[V], const int (&n)[V], int kind, const Place<32>& pl, int warps, float n_warp, int C, float inv_c, float4* room,
                                        float& mean, float& m2) {
    f2 dev = two(0.f);
    if (kind == kRms) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) dev = fma2(f[v].p[i], f[v].p[i], dev);      // channels past the end are 0
        mean = 0.f;
        m2 = lanes_sum<32>(sum_of(dev));
        if (warps > 1) {
            if ((threadIdx.x & 31) == 0) room[pl.warp].y = m2;
            slot_sync(pl.slot, pl.stride);
            m2 = 0.f;
            for (int w = 0; w < warps; ++w) m2 += room[w].y;
        }
        return;
    }
    f2 sum = two(0.f);
#pragma unroll
    for (int v = 0; v < V; ++v) sum = add2(sum, add2(add2(f[v].p[0], f[v].p[1]), add2(f[v].p[2], f[v].p[3])));
    mean = lanes_sum<32>(sum_of(sum)) * (warps == 1 ? inv_c : 1.f / fmaxf(n_warp, 1.f));
    const f2 minus = two(-mean);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (n[v] == kGroup) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { const f2 d = add2(f[v].p[i], minus); dev = fma2(d, d, dev); }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                one_each(add2(f[v].p[i], minus), lo, hi);
                const f2 d = two(2 * i < n[v] ? lo : 0.f, 2 * i + 1 < n[v] ? hi : 0.f);
                dev = fma2(d, d, dev);
            }
        }
    }
    m2 = lanes_sum<32>(sum_of(dev));
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) room[pl.warp] = make_float4(mean, m2, n_warp, 0.f);
        slot_sync(pl.slot, pl.stride);
        const float4 w0 = room[0];       // around the first warp's mean, from which the others differ by the row's spread at most
        float t1 = 0.f, t2 = w0.y;
        for (int w = 1; w < warps; ++w) {
            const float4 q = room[w];
            const float e = q.x - w0.x, ne = q.z * e;
            t1 += ne;
            t2 += fmaf(ne, e, q.y);
        }
        t1 *= inv_c;
        mean = w0.x + t1;
        m2 = fmaf(-float(C) * t1, t1, t2);
        m2 = m2 < 0.f ? 0.f : m2;        // not fmaxf, which takes 0 for the NaN of a row that is not finite
        if (!isfinite(mean)) {           // infinite or NaN, as the channels' sum is
            mean = 0.f;
            for (int w = 0; w < warps; ++w) mean = fmaf(room[w].z * inv_c, room[w].x, mean);
        }
    }
}

// Squares that fp32 cannot sum up, an infinity's among them, have no deviation: NaN, as a row with a NaN has, and not the 0 that 1 / sqrt(infinity) is, which would leave a row of zeros.
__device__ __forceinline__ float rstd_of(float m2, float inv_c, float eps) {
    const float v = fmaf(m2, inv_c, eps);
    return isfinite(v) ? rsqrtf(v) : __uint_as_float(0x7FC00000u);
}

__device__ __forceinline__ float warp_channels(int C, int warp, int col_step, int V) {
    float n = 0.f;
    for (int v = 0; v < V; ++v) n += float(min(max(C - v * col_step - warp * 32 * kGroup, 0), 32 * kGroup));
    return n;
}

// One CTA takes a run of the rows of one batch entry, a slot one row at a time.
template <int V, bool RF, bool XF, bool YF>
__global__ void __launch_bounds__(kThreads, 1) block_forward_kernel(const Args2 a) {
    extern __shared__ float4 smem[];                              // tables of factors, then the stages
    __shared__ float4 part[2][2][kWarps];
    const Place<32> pl(a.warps);
    const int b = blockIdx.y, groups = (a.C + kGroup - 1) / kGroup;
    const int r0 = int(int64_t(blockIdx.x) * a.N / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.N / a.chunks);
    const int col0 = kGroup * pl.at, col_step = kGroup * pl.stride;
    int n[V];
#pragma unroll
    for (int v = 0; v < V; ++v) n[v] = min(max(a.C - col0 - v * col_step, 0), kGroup);
    const bool has_a1 = a.w1 || a.gate, has_c1 = a.b1, has_a2 = a.w2 || a.scale, has_c2 = a.b2 || a.shift;
    const Table ta1(smem, groups), tc1(smem + 2 * groups, groups), ta2(smem + 4 * groups, groups), tc2(smem + 6 * groups, groups);
    const uint32_t ring = uint32_t(__cvta_generic_to_shared(smem)) + uint32_t(groups) * 128u;
    const uint32_t r_bytes = uint32_t(V * (RF ? 2 : 1)) * blockDim.x * 16u, stage = r_bytes + uint32_t(V * (XF ? 2 : 1)) * blockDim.x * 16u;
    const Stage<RF, V, 32> in_r(pl.at);
    const Stage<XF, V, 32> in_x(pl.at);
    const char* r = static_cast<const char*>(a.r) + (b * a.rs[0] + in_r.col) * (RF ? 4 : 2);
    const char* x = static_cast<const char*>(a.x) + (b * a.xs[0] + in_x.col) * (XF ? 4 : 2);
    const int left_r = (a.C - in_r.col) * (RF ? 4 : 2), left_x = (a.C - in_x.col) * (XF ? 4 : 2);
    char* out_s = static_cast<char*>(a.s) + (b * a.ss[0] + col0) * (RF ? 4 : 2);
    char* out_y = static_cast<char*>(a.y) + (b * a.ys[0] + col0) * (YF ? 4 : 2);
    int ahead = r0 + pl.slot;
    grid_launch_dependents();
    grid_wait();                         // launched while the kernel ahead drains: nothing of global memory is touched before this
    auto fetch = [&](int s) {
        const bool on = ahead < r1;
        in_r.copy(ring + uint32_t(s) * stage, r + int64_t(ahead) * a.rs[1] * (RF ? 4 : 2), left_r, col_step, on);
        in_x.copy(ring + uint32_t(s) * stage + r_bytes, x + int64_t(ahead) * a.xs[1] * (XF ? 4 : 2), left_x, col_step, on);
        copies_commit();
        ahead += pl.slots;
    };
    for (int s = 0; s < a.stages; ++s) fetch(s);
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
        float ka[8], kc[8];
        const int left = min(a.C - g * kGroup, kGroup);
        if (has_a1 || has_c1) { factors1(a, b, g * kGroup, left, ka, kc, has_c1); ta1.keep(g, ka); if (has_c1) tc1.keep(g, kc); }
        if (has_a2 || has_c2) { factors2(a, b, g * kGroup, left, ka, kc, has_c2); ta2.keep(g, ka); if (has_c2) tc2.keep(g, kc); }
    }
    __syncthreads();
    const int turns = (r1 - r0 + pl.slots - 1) / pl.slots;
    const float n_warp = warp_channels(a.C, pl.warp, col_step, V);
    int flip = 0, s = 0;
    for (int turn = 0, row = r0 + pl.slot; turn < turns; ++turn, row += pl.slots) {
        copies_wait(a.stages - 1);
        if (RF || XF) __syncwarp();      // the other lanes' copies too
        const uint32_t at = ring + uint32_t(s) * stage;
        Eight f[V];
        float mean1 = 0.f, rstd1 = 1.f, mean2, rstd2, m2;
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = in_x.read(at + r_bytes, v);
        if (a.post != kNone) {
            moments<V>(f, n, a.post, pl, a.warps, n_warp, a.C, a.inv_c, &part[flip][0][pl.slot * a.warps], mean1, m2);
            rstd1 = rstd_of(m2, a.inv_c, a.eps1);
        }
        {
            const f2 minus = two(-mean1), rs = two(rstd1), al = two(a.alpha);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int g = min(pl.at + v * pl.stride, groups - 1);
                const Eight res = in_r.read(at, v);
                const Eight ka = has_a1 ? ta1.kept(g) : Eight{}, kc = has_c1 ? tc1.kept(g) : Eight{};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 t = mul2(add2(f[v].p[i], minus), rs);
                    if (has_a1) t = mul2(t, ka.p[i]);
                    if (has_c1) t = add2(t, kc.p[i]);
                    f[v].p[i] = fma2(res.p[i], al, t);
                }
                if (n[v] < kGroup) {     // channels past the end are 0 for the second norm
                    float q[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) one_each(f[v].p[i], q[2 * i], q[2 * i + 1]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = i < n[v] ? q[i] : 0.f;
                    f[v] = eight_of(q);
                }
            }
        }
        if (RF || XF) __syncwarp();
        fetch(s);                        // into the place just read
        if (++s == a.stages) s = 0;
        const bool on = row < r1;
        if (on) {
            const int64_t so = int64_t(row) * a.ss[1];
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (n[v] > 0) store_eight<RF>(out_s, so + v * col_step, f[v], n[v], a.wide_s);
        }
        moments<V>(f, n, a.pre, pl, a.warps, n_warp, a.C, a.inv_c, &part[flip][1][pl.slot * a.warps], mean2, m2);
        rstd2 = rstd_of(m2, a.inv_c, a.eps2);
        if (on) {
            if (a.stats && pl.at == 0) {
                const int64_t so = int64_t(b) * a.N + row, all = int64_t(a.B) * a.N;
                a.stats[so] = mean1; a.stats[all + so] = rstd1; a.stats[2 * all + so] = mean2; a.stats[3 * all + so] = rstd2;
            }
            const int64_t yo = int64_t(row) * a.ys[1];
            const f2 minus = two(-mean2), rs = two(rstd2);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (n[v] == 0) continue;
                const int g = pl.at + v * pl.stride;
                const Eight ka = has_a2 || has_c2 ? ta2.kept(g) : Eight{}, kc = has_c2 ? tc2.kept(g) : Eight{};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 t = mul2(add2(f[v].p[i], minus), rs);
                    if (has_c2) t = fma2(t, ka.p[i], kc.p[i]);
                    else if (has_a2) t = mul2(t, ka.p[i]);
                    f[v].p[i] = t;
                }
                store_eight<YF>(out_y, yo + v * col_step, f[v], n[v], a.wide_y);
            }
        }
        flip ^= 1;                       // the next row's shares go to the other half: no barrier between a row's last look and the next one's first write
    }
    copies_wait(0);
}

// Sums of two values over a slot's warps.  Within a warp the first step hands one value to the lane half across and takes the other from it, so that two sums take five
// exchanges: the first ends up in the lanes below 16, the second in those above.
__device__ __forceinline__ void slot_sums(float& s1, float& s2, const Place<32>& pl, int warps, float2* room) {
    const int lane = threadIdx.x & 31;
    float s = (lane & 16 ? s2 : s1) + __shfl_xor_sync(0xffffffffu, lane & 16 ? s1 : s2, 16);
#pragma unroll
    for (int m = 8; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    if (warps == 1) {
        s1 = __shfl_sync(0xffffffffu, s, 0);
        s2 = __shfl_sync(0xffffffffu, s, 16);
        return;
    }
    if ((lane & 15) == 0) reinterpret_cast<float*>(room + pl.warp)[lane >> 4] = s;
    slot_sync(pl.slot, pl.stride);
    s1 = 0.f; s2 = 0.f;
    for (int w = 0; w < warps; ++w) { const float2 q = room[w]; s1 += q.x; s2 += q.y; }
}

// dR, dX, and the CTA's partial rows of the four sums.  The row lies in shared memory and its values are read there as often as they are needed: registers hold the sums
// per channel.  Bound by issue slots (51 % busy) and the chains between a row's two means as much as by memory; measured and not kept (32760 x 1536, 198 us as it is): both
// means from one round of eight sums 243, 8 channels per lane instead of 16 and twice the warps 225 to 230, all of the row in registers 230, pieces of 4 channels 347.
template <int V, bool RF, bool XF, bool YF>
__global__ void __launch_bounds__(kThreads, 1) block_backward_kernel(const Args2 a) {
    extern __shared__ float4 smem[];                              // tables, then the stages, which the slots' sums use afterwards
    __shared__ float2 part[2][2][kWarps];
    const Place<32> pl(a.warps);
    const int b = blockIdx.y, groups = (a.C + kGroup - 1) / kGroup;
    const int r0 = int(int64_t(blockIdx.x) * a.N / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.N / a.chunks);
    const int col0 = kGroup * pl.at, col_step = kGroup * pl.stride;
    int n[V];
    Eight P1[V], S1[V], P2[V], S2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        n[v] = min(max(a.C - col0 - v * col_step, 0), kGroup);
#pragma unroll
        for (int i = 0; i < 4; ++i) { P1[v].p[i] = two(0.f); S1[v].p[i] = two(0.f); P2[v].p[i] = two(0.f); S2[v].p[i] = two(0.f); }
    }
    const bool has1 = a.w1 || a.gate, has2 = a.w2 || a.scale;
    const Table t1(smem, groups), t2(smem + 2 * groups, groups);
    float4* stages = smem + 4 * groups;
    const uint32_t ring = uint32_t(__cvta_generic_to_shared(stages));
    // dy, s, ds, x one behind the other
    const uint32_t y_bytes = uint32_t(V * (YF ? 2 : 1)) * blockDim.x * 16u, r_bytes = uint32_t(V * (RF ? 2 : 1)) * blockDim.x * 16u;
    const uint32_t at_s = y_bytes, at_ds = at_s + r_bytes, at_x = at_ds + r_bytes, stage = at_x + uint32_t(V * (XF ? 2 : 1)) * blockDim.x * 16u;
    const Stage<RF, V, 32> in_r(pl.at);
    const Stage<XF, V, 32> in_x(pl.at);
    const Stage<YF, V, 32> in_y(pl.at);
    const char* dy = static_cast<const char*>(a.dy) + (b * a.dys[0] + in_y.col) * (YF ? 4 : 2);
    const char* sv = static_cast<const char*>(a.s) + (b * a.ss[0] + in_r.col) * (RF ? 4 : 2);
    const char* ds = static_cast<const char*>(a.r ? a.r : a.s) + (b * (a.r ? a.rs[0] : 0) + in_r.col) * (RF ? 4 : 2);      // no ds: nothing is copied
    const char* x = static_cast<const char*>(a.x) + (b * a.xs[0] + in_x.col) * (XF ? 4 : 2);
    const int left_r = (a.C - in_r.col) * (RF ? 4 : 2), left_x = (a.C - in_x.col) * (XF ? 4 : 2), left_y = (a.C - in_y.col) * (YF ? 4 : 2);
    char* dr = static_cast<char*>(a.dr) + (b * a.drs[0] + col0) * (RF ? 4 : 2);
    char* dx = static_cast<char*>(a.dx) + (b * a.dxs[0] + col0) * (XF ? 4 : 2);
    int ahead = r0 + pl.slot, after = ahead;
    grid_launch_dependents();
    grid_wait();
    auto fetch = [&](int s) {
        const bool on = ahead < r1;
        const uint32_t to = ring + uint32_t(s) * stage;
        in_y.copy(to, dy + int64_t(ahead) * a.dys[1] * (YF ? 4 : 2), left_y, col_step, on);
        in_r.copy(to + at_s, sv + int64_t(ahead) * a.ss[1] * (RF ? 4 : 2), left_r, col_step, on);
        in_r.copy(to + at_ds, a.r ? ds + int64_t(ahead) * a.rs[1] * (RF ? 4 : 2) : ds, left_r, col_step, on && a.r);
        in_x.copy(to + at_x, x + int64_t(ahead) * a.xs[1] * (XF ? 4 : 2), left_x, col_step, on);
        copies_commit();
        ahead += pl.slots;
    };
    const int64_t all = int64_t(a.B) * a.N;
    float nm1 = 0.f, nr1 = 0.f, nm2 = 0.f, nr2 = 0.f;
    auto stats = [&]() {
        if (after < r1) {
            const float* p = a.stats + int64_t(b) * a.N + after;
            nm1 = p[0]; nr1 = p[all]; nm2 = p[2 * all]; nr2 = p[3 * all];
        }
        after += pl.slots;
    };
    for (int s = 0; s < a.stages; ++s) fetch(s);
    stats();
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
        float ka[8], kc[8];
        const int left = min(a.C - g * kGroup, kGroup);
        if (has1) { factors1(a, b, g * kGroup, left, ka, kc, false); t1.keep(g, ka); }
        if (has2) { factors2(a, b, g * kGroup, left, ka, kc, false); t2.keep(g, ka); }
    }
    __syncthreads();
    const int turns = (r1 - r0 + pl.slots - 1) / pl.slots;
    int flip = 0, s = 0;
    for (int turn = 0, row = r0 + pl.slot; turn < turns; ++turn, row += pl.slots) {
        // what a norm that does not exist has is not taken from the statistics
        const f2 minus1 = two(a.post == kLayer ? -nm1 : 0.f), rs1 = two(a.post == kNone ? 1.f : nr1), minus2 = two(a.pre == kLayer ? -nm2 : 0.f), rs2 = two(nr2);
        stats();
        copies_wait(a.stages - 1);
        __syncwarp();                    // the other lanes' copies too
        const uint32_t at = ring + uint32_t(s) * stage;
        const bool on = row < r1;
        f2 u1 = two(0.f), u2 = two(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Eight d = in_y.read(at, v);
            Eight h = in_r.read(at + at_s, v);
            const Eight ka = has2 ? t2.kept(min(pl.at + v * pl.stride, groups - 1)) : Eight{};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h.p[i] = mul2(add2(h.p[i], minus2), rs2);
                P2[v].p[i] = fma2(d.p[i], h.p[i], P2[v].p[i]);     // channels and rows past the end: dy = 0
                S2[v].p[i] = add2(S2[v].p[i], d.p[i]);
                const f2 t = has2 ? mul2(d.p[i], ka.p[i]) : d.p[i];
                u1 = add2(u1, t);
                u2 = fma2(t, h.p[i], u2);
            }
        }
        float m1 = sum_of(u1), m2 = sum_of(u2);
        slot_sums(m1, m2, pl, a.warps, &part[flip][0][pl.slot * a.warps]);
        const f2 c1 = two(a.pre == kLayer ? -m1 * a.inv_c : 0.f), c2 = two(-m2 * a.inv_c), al = two(a.alpha);
        Eight G[V];
        u1 = two(0.f); u2 = two(0.f);
        const int64_t ro = int64_t(row) * a.drs[1];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int g = min(pl.at + v * pl.stride, groups - 1);
            {
                const Eight d = in_y.read(at, v), e = in_r.read(at + at_ds, v);
                Eight h = in_r.read(at + at_s, v);
                const Eight ka = has2 ? t2.kept(g) : Eight{};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h.p[i] = mul2(add2(h.p[i], minus2), rs2);
                    const f2 t = has2 ? fma2(d.p[i], ka.p[i], c1) : add2(d.p[i], c1);
                    G[v].p[i] = fma2(rs2, fma2(h.p[i], c2, t), e.p[i]);
                }
                if (n[v] < kGroup || !on) {       // past the end: nothing
                    float q[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) one_each(G[v].p[i], q[2 * i], q[2 * i + 1]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = on && i < n[v] ? q[i] : 0.f;
                    G[v] = eight_of(q);
                }
            }
            if (on && n[v] > 0) {
                Eight o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o.p[i] = mul2(G[v].p[i], al);
                store_eight<RF>(dr, ro + v * col_step, o, n[v], a.wide_s);
            }
            Eight h = in_x.read(at + at_x, v);
            const Eight ka = has1 ? t1.kept(g) : Eight{};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h.p[i] = mul2(add2(h.p[i], minus1), rs1);
                P1[v].p[i] = fma2(G[v].p[i], h.p[i], P1[v].p[i]);
                S1[v].p[i] = add2(S1[v].p[i], G[v].p[i]);
                const f2 q = has1 ? mul2(G[v].p[i], ka.p[i]) : G[v].p[i];
                G[v].p[i] = q;
                u1 = add2(u1, q);
                u2 = fma2(q, h.p[i], u2);
            }
        }
        const int64_t xo = int64_t(row) * a.dxs[1];
        if (a.post == kNone) {
            if (on) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (n[v] > 0) store_eight<XF>(dx, xo + v * col_step, G[v], n[v], a.wide_dx);
            }
        } else {
            m1 = sum_of(u1); m2 = sum_of(u2);
            slot_sums(m1, m2, pl, a.warps, &part[flip][1][pl.slot * a.warps]);
            const f2 e1 = two(a.post == kLayer ? -m1 * a.inv_c : 0.f), e2 = two(-m2 * a.inv_c);
            if (on) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (n[v] == 0) continue;
                    Eight h = in_x.read(at + at_x, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        h.p[i] = mul2(add2(h.p[i], minus1), rs1);
                        G[v].p[i] = mul2(rs1, fma2(h.p[i], e2, add2(G[v].p[i], e1)));
                    }
                    store_eight<XF>(dx, xo + v * col_step, G[v], n[v], a.wide_dx);
                }
            }
        }
        __syncwarp();
        fetch(s);                        // into the place just read
        if (++s == a.stages) s = 0;
        flip ^= 1;
    }
    copies_wait(0);
    if (!a.part) return;
    float* out = a.part + (int64_t(b) * a.chunks + blockIdx.x) * 4 * a.C;
    // The slots of the CTA hold sums of the same channels: one after the other in shared memory (where the stages were), added in the order of the slots.
    float* sums = reinterpret_cast<float*>(stages);
    const int width = pl.stride * V * kGroup;
#pragma unroll
    for (int which = 0; which < 4; ++which) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Eight& e = which == 0 ? P1[v] : which == 1 ? S1[v] : which == 2 ? P2[v] : S2[v];
            float4* to = reinterpret_cast<float4*>(sums + pl.slot * width + col0 + v * col_step);
            float p[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) one_each(e.p[i], p[2 * i], p[2 * i + 1]);
            to[0] = make_float4(p[0], p[1], p[2], p[3]);
            to[1] = make_float4(p[4], p[5], p[6], p[7]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            float t = 0.f;
            for (int k = 0; k < pl.slots; ++k) t += sums[k * width + c];
            out[which * a.C + c] = t;
        }
    }
}

struct ReduceArgs2 {
    const float* part;                   // [B * chunks][4][C]
    const void* w1; const void* b1; const void* gate; const void* w2; const void* b2; const void* scale;
    float* dw1; float* db1; float* dgate; float* dw2; float* db2; float* dshift; float* dscale;      // or NULL
    int64_t gate_stride, scale_stride;
    int B, chunks, C, w_f32, mod_f32;
};

// 32 channels per CTA; 16 warps share the partial rows of an entry, and their shares are added in order.
static __global__ void __launch_bounds__(32 * kReduceWarps) block_reduce_kernel(const ReduceArgs2 a) {
    __shared__ float sums[4][kReduceWarps][32];
    grid_launch_dependents();
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const bool on = c < a.C;
    auto param = [&](const void* p, int64_t i, int f32) { return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); };
    auto of = [&](const void* p, float other) { return on && p ? param(p, c, a.w_f32) : other; };
    const float w1 = of(a.w1, 1.f), b1 = of(a.b1, 0.f), w2 = of(a.w2, 1.f), b2 = of(a.b2, 0.f);
    float dw1 = 0.f, db1 = 0.f, dw2 = 0.f, db2 = 0.f;
    for (int b = 0; b < a.B; ++b) {
        float t[4] = {0.f, 0.f, 0.f, 0.f};
        const float* row = a.part + int64_t(b) * a.chunks * 4 * a.C + c;
        if (on)
#pragma unroll 2
            for (int k = warp; k < a.chunks; k += kReduceWarps)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[i] += row[(int64_t(k) * 4 + i) * a.C];
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[i][warp][lane] = t[i];
        __syncthreads();
        if (warp == 0 && on) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t[i] = 0.f;
#pragma unroll
                for (int k = 0; k < kReduceWarps; ++k) t[i] += sums[i][k][lane];
            }
            const float gate = a.gate ? param(a.gate, b * a.gate_stride + c, a.mod_f32) : 1.f, k2 = a.scale ? 1.f + param(a.scale, b * a.scale_stride + c, a.mod_f32) : 1.f;
            dw1 = fmaf(gate, t[0], dw1);
            db1 = fmaf(gate, t[1], db1);
            dw2 = fmaf(k2, t[2], dw2);
            db2 = fmaf(k2, t[3], db2);
            const int64_t at = int64_t(b) * a.C + c;
            if (a.dgate) a.dgate[at] = fmaf(w1, t[0], b1 * t[1]);
            if (a.dscale) a.dscale[at] = fmaf(w2, t[2], b2 * t[3]);
            if (a.dshift) a.dshift[at] = t[3];
        }
        __syncthreads();
    }
    if (warp == 0 && on) {
        if (a.dw1) a.dw1[c] = dw1;
        if (a.db1) a.db1[c] = db1;
        if (a.dw2) a.dw2[c] = dw2;
        if (a.db2) a.db2[c] = db2;
    }
}

// ---- host side ------------------------------------------------------------------------------------
struct Form2 { int warps, v, threads; };
// bytes of shared memory of a CTA: tables, one stage
inline int table2_bytes(int C, bool backward) { return ceil_div(C, kGroup) * (backward ? 64 : 128); }
inline int stage2_bytes(const Form2& f, bool backward, bool rf, bool xf, bool yf) {
    return f.v * f.threads * 16 * ((rf ? 2 : 1) * (backward ? 2 : 1) + (xf ? 2 : 1) + (backward ? (yf ? 2 : 1) : 0));
}
// Warps per row, groups of 8 channels per lane, threads of a CTA (whatever the types are: the workspace goes by it).  The backward kernel keeps four sums per channel
// in registers.  As many slots as 16 warps give and shared memory holds beside the tables.
inline Form2 form2_of(int C, bool backward) {
    const int groups = ceil_div(C, kGroup);
    Form2 f;
    if (backward) { f.warps = ceil_div(groups, 64); f.v = groups <= 32 ? 1 : 2; }
    else if (groups <= 64) { f.warps = 1; f.v = 2; }
    else { f.warps = ceil_div(groups, 128); f.v = std::max(3, ceil_div(groups, 32 * f.warps)); }
    f.threads = 32 * f.warps;
    const int slot = stage2_bytes(f, backward, true, true, true);
    f.threads *= std::max(1, std::min(kWarps / f.warps, (kSmemPerSm - 2048 - table2_bytes(C, backward)) / slot));
    return f;
}
inline int ctas2_per_sm(const Form2& f, int C, bool backward) {
    const int smem = kSmemPerSm / (table2_bytes(C, backward) + stage2_bytes(f, backward, true, true, true) + 2048);
    return std::max(1, std::min(kThreads / f.threads, smem));
}
// CTAs per batch entry, the same for each and not more than there are rows for: all of them one wave, but for entries that outnumber the places.  Entries that do not divide the places leave
// some empty (32760 x 1536 and the like, us: 30000 rows in 1 entry 99 forward, 181 backward; in 50 entries 139, 298; in 75 180, 391).
inline int chunks2_of(const Form2& f, int B, int C, int64_t rows, bool backward) {
    const int64_t slots = f.threads / (32 * f.warps), want = std::max<int64_t>(1, int64_t(148) * ctas2_per_sm(f, C, backward) / B);
    return int(std::min<int64_t>(want, (rows + slots - 1) / slots));
}

// The backward kernel has a few registers more than there are; what shared memory leaves is the L1 cache that holds them (all of it taken for stages: 32760 x 1536 207 us, 198
// so).
constexpr int kBwdSmem = 160 * 1024;
template <int V, bool BWD>
inline cudaError_t launch2_types(Args2 a, const Form2& f, bool rf, bool xf, bool yf, cudaStream_t stream) {
    const int slots = f.threads / (32 * f.warps), turns = ceil_div(ceil_div(a.N, a.chunks), slots);
    const int tables = table2_bytes(a.C, BWD), stage = stage2_bytes(f, BWD, rf, xf, yf), sums = BWD ? f.threads * V * kGroup * 4 : 0;
    a.warps = f.warps;
    a.stages = std::max(1, std::min({kMostStages, ((BWD ? kBwdSmem : kSmemPerSm) / ctas2_per_sm(f, a.C, BWD) - 2048 - tables) / stage, turns}));
    const int smem = tables + std::max(a.stages * stage, sums);
    cudaError_t e = cudaSuccess;
    static SmemAllowed allowed[8];       // of the eight kernels below
    auto run = [&](void (*kernel)(Args2)) {
        if (smem > 40 * 1024) {          // more than a kernel may take unasked, with its static part
            const unsigned long long ctx = context_id();
            SmemAllowed& at = allowed[4 * rf + 2 * xf + yf];
            if (!at.has(ctx)) {
                e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm);
                if (e != cudaSuccess) return;
                at.add(ctx);
            }
        }
        e = launch_dependent(kernel, dim3(unsigned(a.chunks), unsigned(a.B)), dim3(unsigned(f.threads)), size_t(smem), stream, a);
    };
#define CARNATOR_BLOCK(RF, XF, YF)                                                                   \
    if (rf == RF && xf == XF && yf == YF) {                                                          \
        if constexpr (BWD) run(block_backward_kernel<V, RF, XF, YF>);                                \
        else run(block_forward_kernel<V, RF, XF, YF>);                                               \
    }
    CARNATOR_BLOCK(false, false, false)
    CARNATOR_BLOCK(false, false, true)
    CARNATOR_BLOCK(false, true, false)
    CARNATOR_BLOCK(false, true, true)
    CARNATOR_BLOCK(true, false, false)
    CARNATOR_BLOCK(true, false, true)
    CARNATOR_BLOCK(true, true, false)
    CARNATOR_BLOCK(true, true, true)
#undef CARNATOR_BLOCK
    return e;
}
template <bool BWD>
inline cudaError_t launch2(const Args2& a, const Form2& f, bool rf, bool xf, bool yf, cudaStream_t stream) {
    if constexpr (BWD) return f.v == 1 ? launch2_types<1, true>(a, f, rf, xf, yf, stream) : launch2_types<2, true>(a, f, rf, xf, yf, stream);
    else return f.v == 2 ? launch2_types<2, false>(a, f, rf, xf, yf, stream) : f.v == 3 ? launch2_types<3, false>(a, f, rf, xf, yf, stream)
                                                                                    : launch2_types<4, false>(a, f, rf, xf, yf, stream);
}

}  // namespace blk
}  // namespace carnator
