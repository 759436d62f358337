// Layer norm over the channels of a token row, with an affine weight and bias and the modulation of a diffusion transformer
// (shift and scale, one row per batch entry), and its gradients.
//   mu = sum x / C,  rstd = (sum (x - mu)^2 / C + eps)^-1/2,  xh = (x - mu) rstd,  y = (xh w + beta)(1 + scale_b) + shift_b
//   a = w (1 + scale_b),  g = dy a,  dx = rstd (g - mean(g) - xh mean(g xh))
//   P_b = sum over the rows of entry b of dy xh,  S_b = sum of dy:
//   dw = sum_b (1 + scale_b) P_b,  dbeta = sum_b (1 + scale_b) S_b,  dscale_b = w P_b + beta S_b,  dshift_b = S_b
// All four vector gradients follow from P_b and S_b, so the backward kernel keeps two sums per channel and entry, whatever of
// weight, bias, shift and scale there is.
//
// A row is read once and stays in the registers of its lanes (8, 16 or 32 lanes of a warp for short rows, a whole CTA for long
// ones), 8 channels per lane and 16-byte access.  The squared deviations are taken around the mean of a warp's own
// channels first and the warps' shares put together by (mean, sum of squares), which loses nothing when the mean is large against the
// spread and needs one barrier per row instead of two.  The sums per channel stay in registers over all rows of a CTA; each CTA leaves
// one partial row, and a second kernel adds them in a fixed order: no atomics, the same bits every time.
#pragma once
#include "common.cuh"

namespace carnator {
namespace norm {

constexpr int kMaxChannels = 16384;      // 512 threads x 4 groups of 8 channels
constexpr int kGroup = 8;                // channels per lane and access

struct Args {
    const void* x; void* y;              // forward: input, output; backward: x and dX
    const void* dy;
    const void* w; const void* beta;     // [C] or NULL
    const void* shift; const void* scale;   // [B, C] or NULL
    const float* mean_in; const float* rstd_in;
    float* mean; float* rstd;            // [B,H,N] or NULL
    float* part;                         // backward: [B * chunks][2][C] partial P and S, or NULL
    // rows of an entry: `inner` of them beside each other, `outer` times (heads and tokens, the smaller stride of x inside)
    int inner, rows, C, chunks;          // rows = outer * inner per batch entry; chunks of rows per batch entry
    int64_t xs[3], ys[3], ds[3];         // element strides of (batch, outer, inner)
    int64_t ss[3];                       // of the statistics
    int64_t shift_stride, scale_stride;  // of their batch axis
    int w_f32, mod_f32;                  // types of weight and bias, of shift and scale
    int vec_ok;                          // parameter vectors may be read 16 bytes at a time
    float eps, inv_c;
};

template <bool F32> struct Raw8 { uint4 q[F32 ? 2 : 1]; };

template <bool F32>
__device__ __forceinline__ Raw8<F32> load_raw(const void* base, int64_t off, int n) {
    Raw8<F32> r;
    if (n >= kGroup) {
        if (F32) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + off);
            r.q[0] = p[0]; r.q[F32 ? 1 : 0] = p[1];
        } else {
            r.q[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + off);
        }
    } else {                             // the row's last channels: what lies behind them is not the row's
        r.q[0] = make_uint4(0, 0, 0, 0); r.q[F32 ? 1 : 0] = make_uint4(0, 0, 0, 0);
        uint32_t t[F32 ? 8 : 4];
#pragma unroll
        for (int i = 0; i < (F32 ? 8 : 4); ++i) t[i] = 0;
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            if (i < n) {
                if (F32) t[F32 ? i : 0] = static_cast<const uint32_t*>(base)[off + i];
                else t[i / 2] |= uint32_t(static_cast<const uint16_t*>(base)[off + i]) << (16 * (i & 1));
            }
        r.q[0] = make_uint4(t[0], t[1], t[2], t[3]);
        if (F32) r.q[F32 ? 1 : 0] = make_uint4(t[F32 ? 4 : 0], t[F32 ? 5 : 0], t[F32 ? 6 : 0], t[F32 ? 7 : 0]);
    }
    return r;
}
__device__ __forceinline__ void bf16x2_to_float(uint32_t v, float& lo, float& hi) {
    lo = __uint_as_float(v << 16);
    hi = __uint_as_float(v & 0xFFFF0000u);
}
template <bool F32>
__device__ __forceinline__ void to_float(const Raw8<F32>& r, float (&v)[8]) {
    if (F32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 q = r.q[F32 ? h : 0];
            v[4 * h] = __uint_as_float(q.x); v[4 * h + 1] = __uint_as_float(q.y);
            v[4 * h + 2] = __uint_as_float(q.z); v[4 * h + 3] = __uint_as_float(q.w);
        }
    } else {
        bf16x2_to_float(r.q[0].x, v[0], v[1]); bf16x2_to_float(r.q[0].y, v[2], v[3]);
        bf16x2_to_float(r.q[0].z, v[4], v[5]); bf16x2_to_float(r.q[0].w, v[6], v[7]);
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t off, const float (&v)[8], int n) {
    if (n >= kGroup) {
        if (F32) {
            float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + off);
            p[0] = make_float4(v[0], v[1], v[2], v[3]);
            p[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + off) =
                make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            if (i < n) {
                if (F32) static_cast<float*>(base)[off + i] = v[i];
                else static_cast<__nv_bfloat16*>(base)[off + i] = __float2bfloat16_rn(v[i]);
            }
    }
}
// 8 values of a parameter vector (weight, bias, shift, scale, gate), which is aligned to its type only unless vec_ok says 16 bytes
__device__ __forceinline__ void load_param8(const void* base, int64_t off, int f32, int vec_ok, int n, float (&v)[8]) {
    if (vec_ok && n >= kGroup) {
        if (f32) to_float(load_raw<true>(base, off, kGroup), v);
        else to_float(load_raw<false>(base, off, kGroup), v);
    } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            v[i] = i >= n ? 0.f : f32 ? static_cast<const float*>(base)[off + i] : __bfloat162float(static_cast<const __nv_bfloat16*>(base)[off + i]);
    }
}

// sum over the LANES lanes that share a row (LANES = 0: over the warp)
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = (LANES ? LANES : 32) / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

constexpr int most_threads(int lanes, int v) { return lanes || v == 1 ? 256 : 512; }      // as form_of gives them

// Where a lane stands: its row slot within the CTA, its place in the row, how many lanes a row has.
template <int LANES>
struct Place {
    int slot, slots, at, stride;
    __device__ __forceinline__ Place() {
        if (LANES) { slot = threadIdx.x / (LANES ? LANES : 1); slots = blockDim.x / (LANES ? LANES : 1); at = threadIdx.x % (LANES ? LANES : 1); stride = LANES; }
        else { slot = 0; slots = 1; at = threadIdx.x; stride = blockDim.x; }
    }
};

// One CTA takes a run of the rows of one batch entry; a slot takes U rows at a time, all of their loads in flight together.
template <int LANES, int V, int U, bool XF, bool YF>
__global__ void __launch_bounds__(most_threads(LANES, V)) norm_forward_kernel(const Args a) {
    __shared__ float part_mean[2][U][32], part_m2[2][U][32];      // LANES = 0: each warp's mean and squared deviations
    const Place<LANES> pl;
    const int b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r0 = int(int64_t(blockIdx.x) * a.rows / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.rows / a.chunks);
    int col[V], n[V];
    float n_own = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        col[v] = kGroup * (v * pl.stride + pl.at);
        n[v] = min(max(a.C - col[v], 0), kGroup);
        n_own += float(n[v]);
    }
    // channels of this warp, and (lane < warps) of warp `lane`
    float n_warp = 0.f, n_of_lane = 0.f;
    if (!LANES) {
        n_warp = lanes_sum<0>(n_own);
        if (lane < (blockDim.x >> 5))
#pragma unroll
            for (int v = 0; v < V; ++v) n_of_lane += float(min(max(a.C - kGroup * (v * int(blockDim.x) + 32 * lane), 0), 32 * kGroup));
    }
    int flip = 0;
    for (int r = r0; r < r1; r += pl.slots * U) {
        Raw8<XF> x[U][V];
        int64_t yo[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = r + u * pl.slots + pl.slot;
            on[u] = row < r1;
            const int o = row / a.inner, i = row - o * a.inner;
            const int64_t xo = b * a.xs[0] + o * a.xs[1] + i * a.xs[2];
            yo[u] = b * a.ys[0] + o * a.ys[1] + i * a.ys[2];
#pragma unroll
            for (int v = 0; v < V; ++v) x[u][v] = load_raw<XF>(a.x, xo + col[v], on[u] ? n[v] : 0);
        }
        float mean[U], m2[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float f[8];
                to_float(x[u][v], f);
                s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            }
            mean[u] = lanes_sum<LANES>(s);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float mu = LANES ? mean[u] * a.inv_c : mean[u] / fmaxf(n_warp, 1.f);
            float q = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float f[8];
                to_float(x[u][v], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = i < n[v] ? f[i] - mu : 0.f;
                    q = fmaf(d, d, q);
                }
            }
            m2[u] = lanes_sum<LANES>(q);
            mean[u] = mu;
        }
        if (!LANES) {
            if (lane == 0)
#pragma unroll
                for (int u = 0; u < U; ++u) { part_mean[flip][u][warp] = mean[u]; part_m2[flip][u][warp] = m2[u]; }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool has = n_of_lane > 0.f;
                const float mw = has ? part_mean[flip][u][lane] : 0.f, qw = has ? part_m2[flip][u][lane] : 0.f;
                mean[u] = lanes_sum<0>(n_of_lane * mw) * a.inv_c;
                const float d = mw - mean[u];
                m2[u] = lanes_sum<0>(has ? fmaf(n_of_lane * d, d, qw) : 0.f);
            }
            flip ^= 1;                   // the next rows' shares go to the other half: one barrier a turn is enough
        }
        float rs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            rs[u] = rsqrtf(fmaf(m2[u], a.inv_c, a.eps));
            if (a.mean && pl.at == 0 && on[u]) {
                const int row = r + u * pl.slots + pl.slot, o = row / a.inner, i = row - o * a.inner;
                const int64_t so = b * a.ss[0] + o * a.ss[1] + i * a.ss[2];
                a.mean[so] = mean[u];
                a.rstd[so] = rs[u];
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (n[v] == 0) continue;
            float ka[8], kc[8];          // y = xh ka + kc
#pragma unroll
            for (int i = 0; i < 8; ++i) { ka[i] = 1.f; kc[i] = 0.f; }
            if (a.w) load_param8(a.w, col[v], a.w_f32, a.vec_ok, n[v], ka);
            if (a.beta) load_param8(a.beta, col[v], a.w_f32, a.vec_ok, n[v], kc);
            if (a.scale) {
                float t[8];
                load_param8(a.scale, b * a.scale_stride + col[v], a.mod_f32, a.vec_ok, n[v], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) { ka[i] = fmaf(ka[i], t[i], ka[i]); kc[i] = fmaf(kc[i], t[i], kc[i]); }
            }
            if (a.shift) {
                float t[8];
                load_param8(a.shift, b * a.shift_stride + col[v], a.mod_f32, a.vec_ok, n[v], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) kc[i] += t[i];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
                to_float(x[u][v], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = fmaf((f[i] - mean[u]) * rs[u], ka[i], kc[i]);
                if (on[u]) store8<YF>(a.y, yo[u] + col[v], f, n[v]);
            }
        }
    }
}

// dX, and the CTA's partial rows of P and S.
template <int LANES, int V, int U, bool XF, bool YF>
__global__ void __launch_bounds__(most_threads(LANES, V)) norm_backward_kernel(const Args a) {
    __shared__ float part[2][U][2][32];
    __shared__ float slots_sum[LANES ? 256 * kGroup * V : 1];
    const Place<LANES> pl;
    const int b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int r0 = int(int64_t(blockIdx.x) * a.rows / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.rows / a.chunks);
    grid_launch_dependents();
    int col[V], n[V];
    float P[V][8], S[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        col[v] = kGroup * (v * pl.stride + pl.at);
        n[v] = min(max(a.C - col[v], 0), kGroup);
#pragma unroll
        for (int i = 0; i < 8; ++i) { P[v][i] = 0.f; S[v][i] = 0.f; }
    }
    int flip = 0;
    for (int r = r0; r < r1; r += pl.slots * U) {
        Raw8<XF> x[U][V];
        Raw8<YF> dy[U][V];
        float mean[U], rs[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = r + u * pl.slots + pl.slot;
            on[u] = row < r1;
            const int o = row / a.inner, i = row - o * a.inner;
            const int64_t xo = b * a.xs[0] + o * a.xs[1] + i * a.xs[2], dyo = b * a.ds[0] + o * a.ds[1] + i * a.ds[2];
            const int64_t so = b * a.ss[0] + o * a.ss[1] + i * a.ss[2];
            mean[u] = on[u] ? a.mean_in[so] : 0.f;
            rs[u] = on[u] ? a.rstd_in[so] : 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[u][v] = load_raw<XF>(a.x, xo + col[v], on[u] ? n[v] : 0);
                dy[u][v] = load_raw<YF>(a.dy, dyo + col[v], on[u] ? n[v] : 0);
            }
        }
        float ka[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ka[v][i] = 1.f;
            if (a.w) load_param8(a.w, col[v], a.w_f32, a.vec_ok, n[v], ka[v]);
            if (a.scale) {
                float t[8];
                load_param8(a.scale, b * a.scale_stride + col[v], a.mod_f32, a.vec_ok, n[v], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) ka[v][i] = fmaf(ka[v][i], t[i], ka[v][i]);
            }
        }
        float m1[U], m2[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float f[8], d[8];
                to_float(x[u][v], f);
                to_float(dy[u][v], d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xh = (f[i] - mean[u]) * rs[u], g = d[i] * ka[v][i];
                    P[v][i] = fmaf(d[i], xh, P[v][i]);      // channels and rows past the end: d = 0
                    S[v][i] += d[i];
                    s1 += g;
                    s2 = fmaf(g, xh, s2);
                }
            }
            m1[u] = lanes_sum<LANES>(s1);
            m2[u] = lanes_sum<LANES>(s2);
        }
        if (!LANES) {
            if (lane == 0)
#pragma unroll
                for (int u = 0; u < U; ++u) { part[flip][u][0][warp] = m1[u]; part[flip][u][1][warp] = m2[u]; }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                m1[u] = lanes_sum<0>(lane < warps ? part[flip][u][0][lane] : 0.f);
                m2[u] = lanes_sum<0>(lane < warps ? part[flip][u][1][lane] : 0.f);
            }
            flip ^= 1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!on[u]) continue;
            const int row = r + u * pl.slots + pl.slot, o = row / a.inner, i0 = row - o * a.inner;
            const int64_t yo = b * a.ys[0] + o * a.ys[1] + i0 * a.ys[2];
            const float c1 = m1[u] * a.inv_c, c2 = m2[u] * a.inv_c;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (n[v] == 0) continue;
                float f[8], d[8];
                to_float(x[u][v], f);
                to_float(dy[u][v], d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xh = (f[i] - mean[u]) * rs[u];
                    f[i] = rs[u] * (fmaf(d[i], ka[v][i], -c1) - xh * c2);
                }
                store8<XF>(a.y, yo + col[v], f, n[v]);
            }
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t(b) * a.chunks + blockIdx.x) * 2 * a.C;
    if (!LANES) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n[v]) { out[col[v] + i] = P[v][i]; out[a.C + col[v] + i] = S[v][i]; }
    } else {                             // the slots of the CTA hold sums of the same channels
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int width = LANES * V * kGroup;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) slots_sum[pl.slot * width + col[v] + i] = which ? S[v][i] : P[v][i];
            __syncthreads();
            for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
                float s = 0.f;
                for (int k = 0; k < pl.slots; ++k) s += slots_sum[k * width + c];
                out[which * a.C + c] = s;
            }
        }
    }
}

struct ReduceArgs {
    const float* part;                   // [B * chunks][2][C]
    const void* w; const void* beta; const void* scale;
    float* dw; float* dbeta;             // [C] or NULL
    float* dshift; float* dscale;        // [B,C] or NULL
    int64_t scale_stride;
    int B, chunks, C, w_f32, mod_f32;
};

// 32 channels per CTA; 16 warps share the partial rows of an entry, and their shares are added in order.
constexpr int kReduceWarps = 16;
__global__ void __launch_bounds__(32 * kReduceWarps) norm_reduce_kernel(const ReduceArgs a) {
    __shared__ float sums[2][kReduceWarps][32];
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const bool on = c < a.C;
    auto param = [&](const void* p, int64_t i, int f32) { return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); };
    const float w = on && a.w ? param(a.w, c, a.w_f32) : 1.f, beta = on && a.beta ? param(a.beta, c, a.w_f32) : 0.f;
    float dw = 0.f, dbeta = 0.f;
    for (int b = 0; b < a.B; ++b) {
        float p = 0.f, s = 0.f;
        const float* row = a.part + int64_t(b) * a.chunks * 2 * a.C + c;
        if (on)
#pragma unroll 4
            for (int k = warp; k < a.chunks; k += kReduceWarps) {
                p += row[int64_t(k) * 2 * a.C];
                s += row[(int64_t(k) * 2 + 1) * a.C];
            }
        sums[0][warp][lane] = p;
        sums[1][warp][lane] = s;
        __syncthreads();
        if (warp == 0 && on) {
            p = 0.f; s = 0.f;
#pragma unroll
            for (int k = 0; k < kReduceWarps; ++k) { p += sums[0][k][lane]; s += sums[1][k][lane]; }
            const float k1 = a.scale ? 1.f + param(a.scale, b * a.scale_stride + c, a.mod_f32) : 1.f;
            dw = fmaf(k1, p, dw);
            dbeta = fmaf(k1, s, dbeta);
            if (a.dscale) a.dscale[int64_t(b) * a.C + c] = fmaf(w, p, beta * s);
            if (a.dshift) a.dshift[int64_t(b) * a.C + c] = s;
        }
        __syncthreads();
    }
    if (warp == 0 && on) {
        if (a.dw) a.dw[c] = dw;
        if (a.dbeta) a.dbeta[c] = dbeta;
    }
}

// ---- host side ------------------------------------------------------------------------------------
// Lanes per row and groups of 8 channels per lane.
struct Form { int lanes, v, threads; };
inline Form form_of(int C) {
    const int groups = ceil_div(C, kGroup);
    if (groups <= 8) return {8, 1, 256};
    if (groups <= 16) return {16, 1, 256};
    if (groups <= 32) return {32, 1, 256};
    if (groups <= 64) return {32, 2, 256};
    if (groups <= 256) return {0, 1, ceil_div(groups, 32) * 32};
    if (groups <= 1024) return {0, 2, ceil_div(groups, 64) * 32};
    return {0, 4, ceil_div(groups, 128) * 32};
}
// CTAs per batch entry.  Not more rows' worth than there are.  The grid is one wave of what an SM holds.
inline int chunks_of(const Form& f, int B, int64_t rows, bool backward) {
    const int per_sm = f.lanes ? (backward ? 3 : 6) : std::max(1, (backward ? 640 : 1280) / f.threads);
    const int64_t slots = f.lanes ? f.threads / f.lanes : 1;
    const int64_t want = std::max<int64_t>(1, (int64_t(148) * per_sm + B - 1) / B);
    return int(std::min<int64_t>(want, (rows + slots - 1) / slots));
}

template <int LANES, int V, int U, bool BWD>
inline cudaError_t launch_types(const Args& a, dim3 grid, int threads, bool xf, bool yf, cudaStream_t stream) {
#define CARNATOR_NORM(XF, YF)                                                                        \
    if (xf == XF && yf == YF) {                                                                      \
        if (BWD) norm_backward_kernel<LANES, V, U, XF, YF><<<grid, threads, 0, stream>>>(a);         \
        else norm_forward_kernel<LANES, V, U, XF, YF><<<grid, threads, 0, stream>>>(a);              \
    }
    CARNATOR_NORM(false, false)
    CARNATOR_NORM(false, true)
    CARNATOR_NORM(true, false)
    CARNATOR_NORM(true, true)
#undef CARNATOR_NORM
    return cudaGetLastError();
}
template <bool BWD>
inline cudaError_t launch(const Args& a, int B, const Form& f, bool xf, bool yf, cudaStream_t stream) {
    const dim3 grid(a.chunks, B);
    switch (f.lanes * 8 + f.v) {
        case 8 * 8 + 1: return launch_types<8, 1, 2, BWD>(a, grid, f.threads, xf, yf, stream);
        case 16 * 8 + 1: return launch_types<16, 1, 2, BWD>(a, grid, f.threads, xf, yf, stream);
        case 32 * 8 + 1: return launch_types<32, 1, 2, BWD>(a, grid, f.threads, xf, yf, stream);
        case 32 * 8 + 2: return launch_types<32, 2, 1, BWD>(a, grid, f.threads, xf, yf, stream);
        case 1: return launch_types<0, 1, 1, BWD>(a, grid, f.threads, xf, yf, stream);
        case 2: return launch_types<0, 2, 1, BWD>(a, grid, f.threads, xf, yf, stream);
        default: return launch_types<0, 4, 1, BWD>(a, grid, f.threads, xf, yf, stream);
    }
}

}  // namespace norm
}  // namespace carnator
