// Layer norm over the channels of a token row, with an affine weight and bias and the modulation of a diffusion transformer
// (shift and scale, one row per batch entry), and its gradients.
//   mu = sum x / C,  rstd = (sum (x - mu)^2 / C + eps)^-1/2,  xh = (x - mu) rstd,  y = (xh w + beta)(1 + scale_b) + shift_b
//   a = w (1 + scale_b),  g = dy a,  dx = rstd (g - mean(g) - xh mean(g xh))
//   P_b = sum over the rows of entry b of dy xh,  S_b = sum of dy:
//   dw = sum_b (1 + scale_b) P_b,  dbeta = sum_b (1 + scale_b) S_b,  dscale_b = w P_b + beta S_b,  dshift_b = S_b
// All four vector gradients follow from P_b and S_b, so the backward kernel keeps two sums per channel and entry, whatever of
// weight, bias, shift and scale there is.
//
// A row is read once: its lanes (8 to 32 of a warp, or up to 16 warps: a "slot") copy it into shared memory ahead of time (cp.async, each lane what it will read
// itself) and work on it in registers, 8 channels per 16-byte access, up to 32 per lane.  Few lanes with many channels each: what a row costs besides its
// channels (places, sums across lanes) is paid per warp, and at 8 channels a lane it took as many instructions as the channels did (75600 x 5120 in bf16,
// 8 channels a lane 510 us).  The squared deviations are taken around the mean of a warp's own channels first and the warps' shares put together by
// (mean, sum of squares), which loses nothing when the mean is large against the spread and needs one barrier per row instead of two.  The sums per
// channel stay in registers over all rows of a slot; each CTA leaves one partial row, and a second kernel adds them in a fixed order: no atomics, the same
// bits every time.
#pragma once
#include "common.cuh"

namespace carnator {
namespace norm {

constexpr int kMaxChannels = 16384;      // 16 warps x 4 groups of 8 channels a lane
constexpr int kGroup = 8;                // channels per lane and access
constexpr int kMostStages = 4;           // rows ahead per slot

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
    int stages, warps;                   // rows on their way per slot, 1 .. kMostStages; warps of a row
    int wide;                            // every row of the output starts on a 32-byte boundary
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

// ---- two fp32 values per instruction ------------------------------------------------------------------
typedef uint64_t f2;
__device__ __forceinline__ f2 two(float lo, float hi) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ f2 two(float v) { return two(v, v); }
__device__ __forceinline__ void one_each(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ float sum_of(f2 v) { float a, b; one_each(v, a, b); return a + b; }
struct Eight { f2 p[4]; };               // 8 channels

__device__ __forceinline__ Eight eight_of(const float (&v)[8]) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.p[i] = two(v[2 * i], v[2 * i + 1]);
    return e;
}
// fp32 rows on 32-byte boundaries (wide): a whole sector per lane
template <bool F32>
__device__ __forceinline__ void store_eight(void* base, int64_t off, const Eight& e, int n, bool wide) {
    if (F32 && wide && n >= kGroup) {
        asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(static_cast<float*>(base) + off), "l"(e.p[0]), "l"(e.p[1]), "l"(e.p[2]), "l"(e.p[3]) : "memory");
        return;
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) one_each(e.p[i], v[2 * i], v[2 * i + 1]);
    store8<F32>(base, off, v, n);
}

// sum over the LANES lanes of a warp that share a row
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

// Where a lane stands.  LANES < 32: several rows per warp; LANES = 32: a row per warp or, `warps` > 1, per so many warps.
template <int LANES>
struct Place {
    int slot, slots, at, stride, warp;   // row slot in the CTA, place in the row, lanes of a row, warp of the row
    __device__ __forceinline__ explicit Place(int warps) {
        stride = LANES * warps;
        slot = threadIdx.x / stride;
        at = threadIdx.x - slot * stride;
        slots = blockDim.x / stride;
        warp = at >> 5;
    }
};
// a barrier of one slot's warps
__device__ __forceinline__ void slot_sync(int slot, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(slot + 1), "r"(threads) : "memory"); }

// A row of the CTA's run, as (outer, inner); steps by the CTA's slots.
struct Row {
    int row, o, i;
    __device__ __forceinline__ Row(const Args& a, int r) : row(r), o(r / a.inner), i(r - (r / a.inner) * a.inner) {}
    __device__ __forceinline__ void step(const Args& a, int slots, int by_o, int by_i) {
        row += slots;
        o += by_o; i += by_i;
        if (i >= a.inner) { i -= a.inner; ++o; }
    }
    __device__ __forceinline__ int64_t off(const int64_t (&st)[3]) const { return o * st[1] + i * st[2]; }
};

// A row on its way into shared memory: 16-byte pieces, those of the CTA's lanes beside each other.  cp.async reads no byte behind the row's last
// channel and fills the piece with zeros.  bf16: a lane copies the 8 channels that it will read.  fp32: the LANES lanes copy their channels in runs of
// whole sectors (a lane's own 32 bytes in two halves would fetch every sector twice) and exchange them in shared memory; piece p lies at
// p ^ (p / 8 & 1), so that reading pieces 2 l and 2 l + 1 has no bank conflict.
template <bool F32, int V, int LANES>
struct Stage {
    uint32_t put[F32 ? 2 : 1], get[F32 ? 2 : 1];         // byte offsets within a stage
    int col;                                             // first channel that this lane copies
    __device__ __forceinline__ explicit Stage(int at) {
        const uint32_t l = threadIdx.x % LANES, seg = threadIdx.x - l;
        if (F32) {
            col = kGroup * (at - int(l)) + 4 * int(l);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                const uint32_t p = h * LANES + l, q = 2 * l + h, to = p ^ (p >> 3 & 1u), from = q ^ (q >> 3 & 1u);
                put[F32 ? h : 0] = ((to / LANES) * blockDim.x + seg + to % LANES) * 16u;
                get[F32 ? h : 0] = ((from / LANES) * blockDim.x + seg + from % LANES) * 16u;
            }
        } else {
            col = kGroup * at;
            put[0] = get[0] = threadIdx.x * 16u;
        }
    }
    static constexpr uint32_t kPieces = F32 ? 2 : 1;
    // `row`: where the lane's first channel lies in this row; `left`: bytes from there to the end of the row.  A copy of no bytes names an address, but reads
    // nothing there.
    __device__ __forceinline__ void copy(uint32_t dst, const char* row, int left, int col_step, bool on) const {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (uint32_t h = 0; h < kPieces; ++h) {
                const int off = (v * col_step + int(h) * 4 * LANES) * (F32 ? 4 : 2), bytes = on ? min(max(left - off, 0), 16) : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + put[F32 ? h : 0] + v * kPieces * blockDim.x * 16u),
                             "l"(row + off), "r"(bytes) : "memory");
            }
    }
    __device__ __forceinline__ Eight read(uint32_t src, int v) const {
        const uint32_t at = src + v * kPieces * blockDim.x * 16u;
        Eight e;
        if (F32) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(e.p[2 * h]), "=l"(e.p[2 * h + 1]) : "r"(at + get[F32 ? h : 0]) : "memory");
        } else {
            uint32_t q[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(at + get[0]) : "memory");
#pragma unroll
            for (int i = 0; i < 4; ++i) { float lo, hi; bf16x2_to_float(q[i], lo, hi); e.p[i] = two(lo, hi); }
        }
        return e;
    }
};
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int behind) {      // all but the last `behind` groups have landed
    switch (behind) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

// Factors per channel, the same for every row of the CTA: in shared memory, the first and the last four channels of the groups apart, so that a warp's
// 16-byte reads have no bank conflict.
struct Table {
    float4* lo; float4* hi;
    __device__ __forceinline__ Table(float4* base, int groups) : lo(base), hi(base + groups) {}
    __device__ __forceinline__ void keep(int g, const float (&v)[8]) const {
        lo[g] = make_float4(v[0], v[1], v[2], v[3]);
        hi[g] = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ Eight kept(int g) const {
        const float4 a = lo[g], b = hi[g];
        Eight e;
        e.p[0] = two(a.x, a.y); e.p[1] = two(a.z, a.w); e.p[2] = two(b.x, b.y); e.p[3] = two(b.z, b.w);
        return e;
    }
};
// ka = weight (1 + scale), kc = bias (1 + scale) + shift of 8 channels
__device__ __forceinline__ void factors(const Args& a, int b, int col, int n, float (&ka)[8], float (&kc)[8], bool offsets) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { ka[i] = 1.f; kc[i] = 0.f; }
    if (a.w) load_param8(a.w, col, a.w_f32, a.vec_ok, n, ka);
    if (offsets && a.beta) load_param8(a.beta, col, a.w_f32, a.vec_ok, n, kc);
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

// Largest CTA of a form (form_of) and registers per thread.  A bf16 row takes half the registers of an fp32 one, so more threads share an SM.
constexpr int row_warps(bool backward, bool xf) { return backward || xf ? 16 : 20; }
constexpr int most_threads(int lanes, int v, bool backward, bool xf) { return v < 3 || lanes < 32 ? 256 : 32 * row_warps(backward, xf); }
// (A register too few is dear where the rows ahead leave the L1 cache little room: 75600 x 5120 in bf16 322 us with 112, 448 with 80 and 12 bytes spilled.)
constexpr int regs_of(int lanes, int v, bool backward, bool xf) {
    return backward ? (v == 1 ? 96 : 128) : xf ? (v == 1 ? 64 : v == 2 ? 96 : 112) : lanes == 32 ? 96 : v == 1 ? 56 : 80;
}

// One CTA takes a run of the rows of one batch entry, a slot one row at a time.
template <int LANES, int V, bool XF, bool YF>
__global__ void __launch_bounds__(most_threads(LANES, V, false, XF)) __maxnreg__(regs_of(LANES, V, false, XF)) norm_forward_kernel(const Args a) {
    constexpr bool kKeep = V < 3;                                 // few factors per lane: in registers, else in the table
    extern __shared__ float4 smem[];                              // tables (V > 2), then the stages
    __shared__ float4 part[2][24];                                // each warp's mean, squared deviations and channels
    const Place<LANES> pl(a.warps);
    const int b = blockIdx.y, groups = (a.C + kGroup - 1) / kGroup;
    const int r0 = int(int64_t(blockIdx.x) * a.rows / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.rows / a.chunks);
    const int col0 = kGroup * pl.at, col_step = kGroup * pl.stride, by_o = pl.slots / a.inner, by_i = pl.slots - by_o * a.inner;
    int n[V];
#pragma unroll
    for (int v = 0; v < V; ++v) n[v] = min(max(a.C - col0 - v * col_step, 0), kGroup);
    const Table ta(smem, groups), tc(smem + 2 * groups, groups);
    const uint32_t ring = uint32_t(__cvta_generic_to_shared(smem)) + (kKeep ? 0u : uint32_t(groups) * 64u);
    const uint32_t stage = uint32_t(V * (XF ? 2 : 1)) * blockDim.x * 16u;
    const Stage<XF, V, LANES> in(pl.at);
    const char* x = static_cast<const char*>(a.x) + (b * a.xs[0] + in.col) * (XF ? 4 : 2);
    const int left_x = (a.C - in.col) * (XF ? 4 : 2);
    char* y = static_cast<char*>(a.y) + (b * a.ys[0] + col0) * (YF ? 4 : 2);

    Row ahead(a, r0 + pl.slot), now(ahead);
    grid_launch_dependents();
    grid_wait();                         // launched while the kernel ahead drains: nothing of global memory is touched before this
    auto fetch = [&](int s) {
        in.copy(ring + uint32_t(s) * stage, x + ahead.off(a.xs) * (XF ? 4 : 2), left_x, col_step, ahead.row < r1);
        copies_commit();
        ahead.step(a, pl.slots, by_o, by_i);
    };
    for (int s = 0; s < a.stages; ++s) fetch(s);
    Eight rka[kKeep ? V : 1], rkc[kKeep ? V : 1];
    if (kKeep) {
#pragma unroll
        for (int v = 0; v < (kKeep ? V : 1); ++v) {
            float ka[8], kc[8];
            factors(a, b, col0 + v * col_step, n[v], ka, kc, true);
            rka[v] = eight_of(ka); rkc[v] = eight_of(kc);
        }
    } else {
        for (int g = threadIdx.x; g < groups; g += blockDim.x) {
            float ka[8], kc[8];
            factors(a, b, g * kGroup, min(a.C - g * kGroup, kGroup), ka, kc, true);
            ta.keep(g, ka); tc.keep(g, kc);
        }
        __syncthreads();
    }
    const int turns = (r1 - r0 + pl.slots - 1) / pl.slots;
    float n_warp = 0.f;                  // channels of this warp, where a row has several
#pragma unroll
    for (int v = 0; v < V; ++v) n_warp += float(min(max(a.C - v * col_step - pl.warp * 32 * kGroup, 0), 32 * kGroup));
    const float inv_n = LANES < 32 || a.warps == 1 ? a.inv_c : 1.f / fmaxf(n_warp, 1.f);
    int flip = 0, s = 0;
    for (int turn = 0; turn < turns; ++turn) {
        copies_wait(a.stages - 1);
        if (XF) __syncwarp();            // the other lanes' copies too
        Eight f[V];
        f2 sum = two(0.f), dev = two(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            f[v] = in.read(ring + uint32_t(s) * stage, v);
            sum = add2(sum, add2(add2(f[v].p[0], f[v].p[1]), add2(f[v].p[2], f[v].p[3])));
        }
        if (XF) __syncwarp();
        fetch(s);                        // into the place just read
        if (++s == a.stages) s = 0;
        float mean = lanes_sum<LANES>(sum_of(sum)) * inv_n;
        f2 minus = two(-mean);
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
        float m2 = lanes_sum<LANES>(sum_of(dev));
        if (LANES == 32 && a.warps > 1) {
            float4* mine = part[flip] + pl.slot * a.warps;
            if ((threadIdx.x & 31) == 0) mine[pl.warp] = make_float4(mean, m2, n_warp, 0.f);
            slot_sync(pl.slot, pl.stride);
            // around the first warp's mean, from which the others differ by the row's spread at most
            const float4 w0 = mine[0];
            float t1 = 0.f, t2 = w0.y;
            for (int w = 1; w < a.warps; ++w) {
                const float4 q = mine[w];
                const float e = q.x - w0.x, ne = q.z * e;
                t1 += ne;
                t2 += fmaf(ne, e, q.y);
            }
            t1 *= a.inv_c;
            mean = w0.x + t1;
            m2 = fmaf(-float(a.C) * t1, t1, t2);
            m2 = m2 < 0.f ? 0.f : m2;    // not fmaxf, which takes 0 for the NaN of a row that is not finite
            if (!isfinite(mean)) {       // infinite or NaN, as the channels' sum is: the differences from an infinite first warp are not
                mean = 0.f;
                for (int w = 0; w < a.warps; ++w) mean = fmaf(mine[w].z * a.inv_c, mine[w].x, mean);
            }
            flip ^= 1;                   // the next row's shares go to the other half: one barrier a row is enough
            minus = two(-mean);
        }
        const float rstd = rsqrtf(fmaf(m2, a.inv_c, a.eps));
        if (now.row < r1) {
            if (a.mean && pl.at == 0) {
                const int64_t so = b * a.ss[0] + now.off(a.ss);
                a.mean[so] = mean;
                a.rstd[so] = rstd;
            }
            const int64_t yo = now.off(a.ys);
            const f2 rs = two(rstd);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (n[v] == 0) continue;
                const int g = pl.at + v * pl.stride;
                const Eight ka = kKeep ? rka[kKeep ? v : 0] : ta.kept(g), kc = kKeep ? rkc[kKeep ? v : 0] : tc.kept(g);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[v].p[i] = fma2(mul2(add2(f[v].p[i], minus), rs), ka.p[i], kc.p[i]);
                store_eight<YF>(y, yo + v * col_step, f[v], n[v], a.wide);
            }
        }
        now.step(a, pl.slots, by_o, by_i);
    }
    copies_wait(0);
}

// dX, and the CTA's partial rows of P and S.
template <int LANES, int V, bool XF, bool YF>
__global__ void __launch_bounds__(most_threads(LANES, V, true, XF)) __maxnreg__(regs_of(LANES, V, true, XF)) norm_backward_kernel(const Args a) {
    constexpr bool kKeep = V < 3;
    extern __shared__ float4 smem[];                              // table (V > 2), then the stages, which the slots' sums use afterwards
    __shared__ float2 part[2][16];
    const Place<LANES> pl(a.warps);
    const int b = blockIdx.y, groups = (a.C + kGroup - 1) / kGroup;
    const int r0 = int(int64_t(blockIdx.x) * a.rows / a.chunks), r1 = int(int64_t(blockIdx.x + 1) * a.rows / a.chunks);
    grid_launch_dependents();
    grid_wait();
    const int col0 = kGroup * pl.at, col_step = kGroup * pl.stride, by_o = pl.slots / a.inner, by_i = pl.slots - by_o * a.inner;
    int n[V];
    Eight P[V], S[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        n[v] = min(max(a.C - col0 - v * col_step, 0), kGroup);
#pragma unroll
        for (int i = 0; i < 4; ++i) { P[v].p[i] = two(0.f); S[v].p[i] = two(0.f); }
    }
    const Table ta(smem, groups);
    float4* stages = smem + (kKeep ? 0 : 2 * groups);
    const uint32_t ring = uint32_t(__cvta_generic_to_shared(stages));
    const uint32_t x_bytes = uint32_t(V * (XF ? 2 : 1)) * blockDim.x * 16u, stage = x_bytes + uint32_t(V * (YF ? 2 : 1)) * blockDim.x * 16u;
    const Stage<XF, V, LANES> in(pl.at);
    const Stage<YF, V, LANES> in_dy(pl.at);
    const char* x = static_cast<const char*>(a.x) + (b * a.xs[0] + in.col) * (XF ? 4 : 2);
    const char* dy = static_cast<const char*>(a.dy) + (b * a.ds[0] + in_dy.col) * (YF ? 4 : 2);
    const int left_x = (a.C - in.col) * (XF ? 4 : 2), left_dy = (a.C - in_dy.col) * (YF ? 4 : 2);
    char* dx = static_cast<char*>(a.y) + (b * a.ys[0] + col0) * (XF ? 4 : 2);

    Row ahead(a, r0 + pl.slot), now(ahead), after(ahead);
    auto fetch = [&](int s) {
        const bool on = ahead.row < r1;
        in.copy(ring + uint32_t(s) * stage, x + ahead.off(a.xs) * (XF ? 4 : 2), left_x, col_step, on);
        in_dy.copy(ring + uint32_t(s) * stage + x_bytes, dy + ahead.off(a.ds) * (YF ? 4 : 2), left_dy, col_step, on);
        copies_commit();
        ahead.step(a, pl.slots, by_o, by_i);
    };
    float next_mean = 0.f, next_rstd = 0.f;
    auto stats = [&]() {
        if (after.row < r1) {
            const int64_t so = b * a.ss[0] + after.off(a.ss);
            next_mean = a.mean_in[so];
            next_rstd = a.rstd_in[so];
        }
        after.step(a, pl.slots, by_o, by_i);
    };
    for (int s = 0; s < a.stages; ++s) fetch(s);
    stats();
    Eight rka[kKeep ? V : 1];
    if (kKeep) {
#pragma unroll
        for (int v = 0; v < (kKeep ? V : 1); ++v) {
            float ka[8], kc[8];
            factors(a, b, col0 + v * col_step, n[v], ka, kc, false);
            rka[v] = eight_of(ka);
        }
    } else {
        for (int g = threadIdx.x; g < groups; g += blockDim.x) {
            float ka[8], kc[8];
            factors(a, b, g * kGroup, min(a.C - g * kGroup, kGroup), ka, kc, false);
            ta.keep(g, ka);
        }
        __syncthreads();
    }
    const int turns = (r1 - r0 + pl.slots - 1) / pl.slots;
    int flip = 0, s = 0;
    for (int turn = 0; turn < turns; ++turn) {
        const f2 minus = two(-next_mean), rs = two(next_rstd);
        stats();
        copies_wait(a.stages - 1);
        if (XF || YF) __syncwarp();      // the other lanes' copies too
        // The row is read from shared memory twice, before and after its sums: registers hold the sums per channel, and keeping the row there too took
        // half of the lanes.
        const uint32_t at = ring + uint32_t(s) * stage;
        auto read = [&](int v, Eight& xh, Eight& g) {
            xh = in.read(at, v);
            g = in_dy.read(at + x_bytes, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) xh.p[i] = mul2(add2(xh.p[i], minus), rs);
        };
        f2 s1 = two(0.f), s2 = two(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Eight ka = kKeep ? rka[kKeep ? v : 0] : ta.kept(min(pl.at + v * pl.stride, groups - 1));
            Eight xh, g;
            read(v, xh, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                P[v].p[i] = fma2(g.p[i], xh.p[i], P[v].p[i]);      // channels and rows past the end: dy = 0
                S[v].p[i] = add2(S[v].p[i], g.p[i]);
                const f2 t = mul2(g.p[i], ka.p[i]);
                s1 = add2(s1, t);
                s2 = fma2(t, xh.p[i], s2);
            }
        }
        float m1 = lanes_sum<LANES>(sum_of(s1)), m2 = lanes_sum<LANES>(sum_of(s2));
        if (LANES == 32 && a.warps > 1) {
            float2* mine = part[flip] + pl.slot * a.warps;
            if ((threadIdx.x & 31) == 0) mine[pl.warp] = make_float2(m1, m2);
            slot_sync(pl.slot, pl.stride);
            m1 = 0.f; m2 = 0.f;
            for (int w = 0; w < a.warps; ++w) { const float2 q = mine[w]; m1 += q.x; m2 += q.y; }
            flip ^= 1;
        }
        if (now.row < r1) {
            const int64_t yo = now.off(a.ys);
            const f2 c1 = two(-m1 * a.inv_c), c2 = two(-m2 * a.inv_c);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (n[v] == 0) continue;
                const Eight ka = kKeep ? rka[kKeep ? v : 0] : ta.kept(pl.at + v * pl.stride);
                Eight xh, g;
                read(v, xh, g);
#pragma unroll
                for (int i = 0; i < 4; ++i) g.p[i] = mul2(rs, fma2(xh.p[i], c2, fma2(g.p[i], ka.p[i], c1)));
                store_eight<XF>(dx, yo + v * col_step, g, n[v], a.wide);
            }
        }
        if (XF || YF) __syncwarp();
        fetch(s);                        // into the place just read
        if (++s == a.stages) s = 0;
        now.step(a, pl.slots, by_o, by_i);
    }
    copies_wait(0);
    if (!a.part) return;
    float* out = a.part + (int64_t(b) * a.chunks + blockIdx.x) * 2 * a.C;
    if (pl.slots == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (n[v] == 0) continue;
            float p[8], q[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { one_each(P[v].p[i], p[2 * i], p[2 * i + 1]); one_each(S[v].p[i], q[2 * i], q[2 * i + 1]); }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n[v]) { out[col0 + v * col_step + i] = p[i]; out[a.C + col0 + v * col_step + i] = q[i]; }
        }
        return;
    }
    // The slots of the CTA hold sums of the same channels: one after the other in shared memory (where the stages were), added in the order of the slots.
    float* sums = reinterpret_cast<float*>(stages);
    const int width = pl.stride * V * kGroup;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float4* at = reinterpret_cast<float4*>(sums + pl.slot * width + col0 + v * col_step);
            float p[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) one_each(which ? S[v].p[i] : P[v].p[i], p[2 * i], p[2 * i + 1]);
            at[0] = make_float4(p[0], p[1], p[2], p[3]);
            at[1] = make_float4(p[4], p[5], p[6], p[7]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            float t = 0.f;
            for (int k = 0; k < pl.slots; ++k) t += sums[k * width + c];
            out[which * a.C + c] = t;
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
    grid_launch_dependents();
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
// Lanes (of a warp) and warps per row, groups of 8 channels per lane, threads of a CTA.
// The backward kernel keeps two sums per channel in registers, so where rows share a warp it has fewer channels per lane.
struct Form { int lanes, warps, v, threads; };
inline Form form_of(int C, bool backward, bool xf) {
    const int groups = ceil_div(C, kGroup);
    if (groups <= 8) return {8, 1, 1, 256};
    if (groups <= 16) return {8, 1, 2, 256};
    if (groups <= 32) return backward ? Form{16, 1, 2, 256} : Form{8, 1, 4, 256};
    if (groups <= 64) return backward ? Form{32, 1, 2, 256} : Form{16, 1, 4, 256};
    // As many slots as a CTA's warps give, which share the table of factors.  Three groups per lane leave the fp32 backward kernel its registers (75600 x
    // 5120: 713 us with four and 36 bytes spilled, 651 with three); bf16 wants four (466 us, with three 547).
    const int warps = ceil_div(groups, backward && xf && groups <= 16 * 96 ? 96 : 128), v = ceil_div(groups, 32 * warps);
    return {32, warps, v < 3 ? 3 : v, 32 * warps * (row_warps(backward, xf) / warps)};
}
constexpr int kSmemPerSm = 220 * 1024;
// bytes of shared memory of a CTA: tables, one stage of rows (fp32, the wider type, unless the types are known)
inline int table_bytes(const Form& f, int C, bool backward) { return f.v < 3 ? 0 : ceil_div(C, kGroup) * (backward ? 32 : 64); }
inline int stage_bytes(const Form& f, bool backward, bool xf, bool yf) { return f.v * f.threads * 16 * ((xf ? 2 : 1) + (backward ? (yf ? 2 : 1) : 0)); }
// CTAs that share an SM: as many as its registers hold and its shared memory does with one stage each.
inline int ctas_per_sm(const Form& f, int C, bool backward, bool xf) {
    const int regs = 65536 / (regs_of(f.lanes, f.v, backward, xf) * f.threads), smem = kSmemPerSm / (table_bytes(f, C, backward) + stage_bytes(f, backward, xf, true) + 2048);
    return std::max(1, std::min({2048 / f.threads, regs, smem}));
}
// CTAs per batch entry: one wave, and not more than there are rows for.
inline int chunks_of(const Form& f, int B, int C, int64_t rows, bool backward, bool xf) {
    const int64_t slots = f.threads / (f.lanes * f.warps);
    const int64_t want = std::max<int64_t>(1, int64_t(148) * ctas_per_sm(f, C, backward, xf) / B);
    return int(std::min<int64_t>(want, (rows + slots - 1) / slots));
}

template <int LANES, int V, bool BWD>
inline cudaError_t launch_types(Args a, dim3 grid, const Form& f, bool xf, bool yf, cudaStream_t stream) {
    const int slots = f.threads / (f.lanes * f.warps), turns = ceil_div(ceil_div(a.rows, a.chunks), slots);
    const int tables = table_bytes(f, a.C, BWD), stage = stage_bytes(f, BWD, xf, yf);
    const int sums = BWD && slots > 1 ? f.threads * V * kGroup * 4 : 0;      // the slots' sums, in the stages' place
    a.warps = f.warps;
    a.stages = std::max(1, std::min({kMostStages, (kSmemPerSm / ctas_per_sm(f, a.C, BWD, xf) - 2048 - tables) / stage, turns}));
    const int smem = tables + std::max(a.stages * stage, sums);
    cudaError_t e = cudaSuccess;
    static SmemAllowed allowed[4];       // of the four kernels below
    auto run = [&](void (*kernel)(Args)) {
        if (smem > 40 * 1024) {          // more than a kernel may take unasked, with its static part
            const unsigned long long ctx = context_id();
            SmemAllowed& at = allowed[2 * xf + yf];
            if (!at.has(ctx)) {
                e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm);
                if (e != cudaSuccess) return;
                at.add(ctx);
            }
        }
        e = launch_dependent(kernel, grid, dim3(f.threads), smem, stream, a);
    };
#define CARNATOR_NORM(XF, YF)                                                                        \
    if (xf == XF && yf == YF) {                                                                      \
        if constexpr (BWD) run(norm_backward_kernel<LANES, V, XF, YF>);                              \
        else run(norm_forward_kernel<LANES, V, XF, YF>);                                             \
    }
    CARNATOR_NORM(false, false)
    CARNATOR_NORM(false, true)
    CARNATOR_NORM(true, false)
    CARNATOR_NORM(true, true)
#undef CARNATOR_NORM
    return e;
}
template <bool BWD>
inline cudaError_t launch(const Args& a, int B, const Form& f, bool xf, bool yf, cudaStream_t stream) {
    const dim3 grid(a.chunks, B);
    if (f.lanes == 8 && f.v == 1) return launch_types<8, 1, BWD>(a, grid, f, xf, yf, stream);
    if (f.lanes == 8 && f.v == 2) return launch_types<8, 2, BWD>(a, grid, f, xf, yf, stream);
    if constexpr (BWD) {
        if (f.lanes == 16) return launch_types<16, 2, BWD>(a, grid, f, xf, yf, stream);
        if (f.v == 2) return launch_types<32, 2, BWD>(a, grid, f, xf, yf, stream);
    } else {
        if (f.lanes == 8) return launch_types<8, 4, BWD>(a, grid, f, xf, yf, stream);
        if (f.lanes == 16) return launch_types<16, 4, BWD>(a, grid, f, xf, yf, stream);
    }
    return f.v == 3 ? launch_types<32, 3, BWD>(a, grid, f, xf, yf, stream) : launch_types<32, 4, BWD>(a, grid, f, xf, yf, stream);
}

}  // namespace norm
}  // namespace carnator
