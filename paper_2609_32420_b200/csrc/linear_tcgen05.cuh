// Matrix products of a layer's projections on the 5th-generation tensor cores, with everything that follows the product in the
// epilogue:   z = x W^T + bias,   y = residual + gate_b act(z)   (and z itself, for the backward pass),
// and the two products of its gradients, dX = dz W and dW = dz^T x.
//
// One kernel, D[m,n] = sum_k A[m,k] B[n,k]; either operand may have its k axis contiguous (K-major: x, W and dz in the forward
// product and dX) or its m / n axis (MN-major: W in dX, both in dW), which only changes the boxes that TMA fetches and the descriptors.
// A pair of CTAs shares a tile of 256 x BN (tcgen05 cta_group::2): each loads 128 rows of A and half of the rows of B, and the product
// of the pair reads both halves, so that an SM stages 32 KB per 64 columns of k where a CTA on its own would stage 48 KB for the same
// flops.  Accumulators: 2 x 256 fp32 columns of tensor memory, so a tile's epilogue runs under the next tile's product.
//
// Warp roles (384 threads, one CTA per SM): warp 0 TMA producer; warp 1 (of the pair's first CTA) MMA issue; warp 2 tensor-memory
// allocation; warps 4-11 epilogue.
// The epilogue stays in registers: a lane holds a row's 32 columns and reads the residual and writes y and z in whole 32-byte sectors of its row.
// (Turned through shared memory, so that a warp's access covers runs of a row, the same bytes cost the product its operands: the ring's writes
// and the reads of the products take nearly all of the 128 bytes a clock that shared memory has.  32760 x 1536 x 8960 with z and
// GELU 754 us that way.)
// Few tiles: 2 or 4 pairs of one cluster take a share of k each and add their partial tiles through distributed shared memory, in
// the order of k: no workspace, no atomics, the same bits every time.
// Every wait on an mbarrier is bounded, as in the attention kernel.
#pragma once
#include <cuda.h>

#include "attn_tcgen05.cuh"
#include "norm.cuh"

namespace carnator {
namespace lin {
using namespace tc;

constexpr int kThreadsTc = 384;
constexpr int kEpiWarps = 8;
constexpr int kTileM = 256;              // rows of a pair's tile
constexpr int kSlab = 64;                // columns of a slab: one 128-byte swizzle row of bf16
constexpr int kMaxStages = 8;
constexpr uint32_t kRingBytes = 225 * 1024;          // stages
constexpr uint32_t kSmemTc = kRingBytes + 512 + 1024;      // barriers, slack to align the base to 1 KB
static_assert(kSmemTc + 256 <= 232448, "shared memory of a CTA");

enum { kActNone = 0, kActGeluTanh = 1, kActGelu = 2, kActSilu = 3 };

// What follows the product.
struct Epilogue {
    void* y; void* z;                    // z: bf16 or NULL
    const void* bias; const void* gate; const void* residual;
    int64_t ys[2], zs[2], rs[2], gate_stride;      // (batch, row)
    int act, y_f32, bias_f32, gate_f32, vec_ok;
    int wide_ok;                         // rows of y, z and residual start on 32-byte boundaries
    int rows_per_gate;                   // rows that share a gate row (batch entries that follow each other evenly are one)
};

struct TcArgs {
    Epilogue e;
    WsHeader* hdr;
    int batches, rows, cols;             // D: rows per batch entry, columns
    int tiles_m, tiles_n, tiles;         // per batch entry; columns; all of them
    int group_m;                         // row tiles that are worked through together, column by column
    int bn;                              // columns of a tile, a multiple of 32 (of 128 where B is MN-major)
    int k_batches, k_tiles;              // k: batch entries (dW) x tiles of 64
    int k_len;                           // k of a batch entry
    int a_slabs, b_slabs;                // MN-major: whole 64-column slabs of the operand, which a tile fetches in one copy where all of its slabs are whole
    int stages, splits;
    int clears;                          // the first product of a call clears its status word
};

__device__ __forceinline__ uint32_t cluster_ctarank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t map_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// What it orders are reads of tensor memory that have completed: CTA scope.  (Releasing at cluster scope waits for the thread's earlier
// stores to global memory.)
__device__ __forceinline__ void arrive_remote(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// the copy lands in this CTA and counts on the barrier of the pair's first CTA
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, uint32_t cluster_bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_load_pair_slabs(uint32_t dst, const CUtensorMap* map, uint32_t cluster_bar, int row, int slab, int batch) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(0), "r"(row), "r"(slab), "r"(batch) : "memory");
}
__device__ __forceinline__ void mma_pair_el(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier at this offset in both CTAs of the pair once every product issued so far has completed
__device__ __forceinline__ void commit_pair_el(uint32_t bar, uint16_t mask) {
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
        ::"r"(bar), "h"(mask) : "memory");
}

// ---- activations ----------------------------------------------------------------------------------
// Value and slope, each from one exponential and one reciprocal (the pipe for these takes 8 clocks for a warp's 32, which bounds the pass that
// computes both for the gradients as soon as it is not memory).
//   silu       z g, g = 1 / (1 + exp(-z));  slope g + z g (1 - g)
//   gelu_tanh  z (1 + tanh u) / 2 = z g, g = 1 / (1 + exp(-2u)), u = A (z + B z^3): no cancellation where tanh is near -1;
//              slope g + 2 z g (1 - g) u', u' = A (1 + 3 B z^2)
//   gelu       z Phi(z); Phi(-a) = exp(-a^2 / 2) (c1 t + .. + c8 t^8), t = 1 / (1 + 0.33 a / sqrt 2), a >= 0, and 1 - Phi(-a) on the other side: the polynomial
//              has the least largest relative error against erfc(x) exp(x^2) / 2 over x = 0 .. 9.6 (8.2e-8; fitted by repeatedly weighted least squares in
//              64 bits), so that values far below zero keep their bits.  Its exponential is the density's.  slope Phi + z exp(-z^2 / 2) / sqrt(2 pi)
// The exponentials and reciprocals are the approximate instructions' (2^-22 of a result or so); an argument's rounding costs 2^-24 of it each time.
constexpr float kGeluA = 0.7978845608028654f, kGeluB = 0.044715f;
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
using norm::f2; using norm::two; using norm::one_each; using norm::add2; using norm::mul2; using norm::fma2;
__device__ __forceinline__ f2 ex2_each(f2 v) { float a, b; one_each(v, a, b); return two(ex2_approx(a), ex2_approx(b)); }
__device__ __forceinline__ f2 rcp_each(f2 v) { float a, b; one_each(v, a, b); return two(rcp_approx(a), rcp_approx(b)); }
__device__ __forceinline__ f2 less_from(f2 v, float from) { return fma2(v, two(-1.f), two(from)); }
// of two arguments, two fp32 values per instruction
template <int ACT>
__device__ __forceinline__ void act_and_slope(f2 z, f2& f, f2& s) {
    if (ACT == kActSilu) {
        const f2 g = rcp_each(add2(ex2_each(mul2(z, two(-kLog2e))), two(1.f)));
        f = mul2(z, g);
        s = fma2(f, less_from(g, 1.f), g);
    } else if (ACT == kActGelu) {
        float lo, hi;
        one_each(z, lo, hi);
        const f2 t = rcp_each(fma2(two(fabsf(lo), fabsf(hi)), two(0.33f * 0.7071067811865476f), two(1.f)));
        const f2 e = ex2_each(mul2(mul2(z, two(-0.5f * kLog2e)), z));
        f2 p = fma2(t, two(-0.0679643637f), two(0.231343965f));
        p = fma2(p, t, two(-0.177719204f));
        p = fma2(p, t, two(0.206270549f));
        p = fma2(p, t, two(0.0225054619f));
        p = fma2(p, t, two(0.100961868f));
        p = fma2(p, t, two(0.0914186282f));
        p = fma2(p, t, two(0.0931830544f));
        const f2 below = mul2(mul2(p, t), e), above = less_from(below, 1.f);
        float b0, b1, a0, a1;
        one_each(below, b0, b1);
        one_each(above, a0, a1);
        const f2 c = two(lo < 0.f ? b0 : a0, hi < 0.f ? b1 : a1);
        f = mul2(z, c);
        s = fma2(mul2(z, two(0.3989422804014327f)), e, c);
    } else if (ACT == kActGeluTanh) {
        const f2 zz = mul2(z, z);
        const f2 u = mul2(z, fma2(zz, two(-2.f * kLog2e * kGeluA * kGeluB), two(-2.f * kLog2e * kGeluA)));
        const f2 g = rcp_each(add2(ex2_each(u), two(1.f)));
        f = mul2(z, g);
        float lo, hi;                    // the square of a z beyond 1.8e19 is infinite, and the factor before it 0
        one_each(zz, lo, hi);
        s = fma2(mul2(f, less_from(g, 1.f)), fma2(two(fminf(lo, 1e30f), fminf(hi, 1e30f)), two(6.f * kGeluA * kGeluB), two(2.f * kGeluA)), g);
    } else {
        f = z; s = two(1.f);
    }
}
template <int ACT>
__device__ __forceinline__ void activation2(float& a, float& b) {
    f2 f, s;
    act_and_slope<ACT>(two(a, b), f, s);
    one_each(f, a, b);
}
template <int ACT>
__device__ __forceinline__ float activation(float z) {
    float a = z, b = z;
    activation2<ACT>(a, b);
    return a;
}
template <int ACT>
__device__ __forceinline__ void activate8(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) activation2<ACT>(v[i], v[i + 1]);
}
__device__ __forceinline__ void activate8(float (&v)[8], int act) {
    switch (act) {
        case kActGeluTanh: activate8<kActGeluTanh>(v); break;
        case kActGelu: activate8<kActGelu>(v); break;
        case kActSilu: activate8<kActSilu>(v); break;
        default: break;
    }
}

// ---- epilogue of 8 columns of one row ---------------------------------------------------------------
struct Columns {                         // what 8 columns share over the rows of a piece
    float bias[8], gate[8];
    int gate_row;
};
__device__ __forceinline__ void columns_begin(const Epilogue& e, Columns& c, int col, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { c.bias[i] = 0.f; c.gate[i] = 1.f; }
    if (e.bias) norm::load_param8(e.bias, col, e.bias_f32, e.vec_ok, n, c.bias);
    c.gate_row = -1;
}
__device__ __forceinline__ void load_residual(const Epilogue& e, int b, int row, int col, int n, norm::Raw8<true>& r) {
    const int64_t off = b * e.rs[0] + row * e.rs[1] + col;
    if (e.y_f32) r = norm::load_raw<true>(e.residual, off, n);
    else r.q[0] = norm::load_raw<false>(e.residual, off, n).q[0];
}
__device__ __forceinline__ void finish(const Epilogue& e, Columns& c, int b, int row, int col, int n, float (&v)[8], const norm::Raw8<true>& res) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += c.bias[i];
    if (e.z) norm::store8<false>(e.z, b * e.zs[0] + row * e.zs[1] + col, v, n);
    activate8(v, e.act);
    if (e.gate) {
        const int g = b + row / e.rows_per_gate;
        if (g != c.gate_row) { norm::load_param8(e.gate, g * e.gate_stride + col, e.gate_f32, e.vec_ok, n, c.gate); c.gate_row = g; }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= c.gate[i];
    }
    if (e.residual) {
        float r[8];
        if (e.y_f32) norm::to_float(res, r);
        else { norm::Raw8<false> h; h.q[0] = res.q[0]; norm::to_float(h, r); }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    const int64_t off = b * e.ys[0] + row * e.ys[1] + col;
    if (e.y_f32) norm::store8<true>(e.y, off, v, n);
    else norm::store8<false>(e.y, off, v, n);
}

// 32 bytes: a whole sector per lane.  No clobber of memory: a residual is read by the lane that writes y over it, before.
struct Sector { uint32_t q[8]; };
// `wide`: it starts on a 32-byte boundary; else on a 16-byte one.
__device__ __forceinline__ Sector load_sector(const void* p, int wide) {
    Sector s;
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(s.q[0]), "=r"(s.q[1]), "=r"(s.q[2]), "=r"(s.q[3]),
                     "=r"(s.q[4]), "=r"(s.q[5]), "=r"(s.q[6]), "=r"(s.q[7]) : "l"(p));
    } else {
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%8];\n\tld.global.v4.b32 {%4, %5, %6, %7}, [%8+16];" : "=&r"(s.q[0]), "=&r"(s.q[1]), "=&r"(s.q[2]), "=&r"(s.q[3]),
                     "=&r"(s.q[4]), "=&r"(s.q[5]), "=&r"(s.q[6]), "=&r"(s.q[7]) : "l"(p));
    }
    return s;
}
__device__ __forceinline__ void store_sector(void* p, const Sector& s, int wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(s.q[0]), "r"(s.q[1]), "r"(s.q[2]), "r"(s.q[3]),
                     "r"(s.q[4]), "r"(s.q[5]), "r"(s.q[6]), "r"(s.q[7]));
    } else {
        asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\tst.global.v4.b32 [%0+16], {%5, %6, %7, %8};" ::"l"(p), "r"(s.q[0]), "r"(s.q[1]), "r"(s.q[2]), "r"(s.q[3]),
                     "r"(s.q[4]), "r"(s.q[5]), "r"(s.q[6]), "r"(s.q[7]));
    }
}
__device__ __forceinline__ Sector pack16(const float (&v)[16]) {
    Sector s;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.q[i] = norm::pack_bf16(v[2 * i], v[2 * i + 1]);
    return s;
}
// 16 values of a parameter vector
__device__ __forceinline__ void load_param16(const void* base, int64_t off, int f32, int vec_ok, float (&v)[16]) {
    float a[8], b[8];
    norm::load_param8(base, off, f32, vec_ok, 8, a);
    norm::load_param8(base, off + 8, f32, vec_ok, 8, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[i] = a[i]; v[8 + i] = b[i]; }
}
// Epilogue of 16 columns of one row, all of them there.  `gate`: the entry's gate row or NULL;
// `res`: the residual's sectors (one of bf16, two of fp32), loaded before.
template <bool YF>
__device__ __forceinline__ void finish16(const Epilogue& e, const void* gate, int64_t gate_off, int64_t y_off, int64_t z_off, int col, float (&v)[16],
                                         const Sector& r0, const Sector& r1) {
    if (e.bias) {
        float t[16];
        load_param16(e.bias, col, e.bias_f32, e.vec_ok, t);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += t[i];
    }
    if (e.z) store_sector(static_cast<__nv_bfloat16*>(e.z) + z_off + col, pack16(v), e.wide_ok);
    switch (e.act) {
        case kActGeluTanh:
#pragma unroll
            for (int i = 0; i < 16; i += 2) activation2<kActGeluTanh>(v[i], v[i + 1]);
            break;
        case kActGelu:
#pragma unroll
            for (int i = 0; i < 16; i += 2) activation2<kActGelu>(v[i], v[i + 1]);
            break;
        case kActSilu:
#pragma unroll
            for (int i = 0; i < 16; i += 2) activation2<kActSilu>(v[i], v[i + 1]);
            break;
        default: break;
    }
    if (gate) {
        float t[16];
        load_param16(gate, gate_off + col, e.gate_f32, e.vec_ok, t);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= t[i];
    }
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (YF) { v[i] += __uint_as_float(r0.q[i]); v[8 + i] += __uint_as_float(r1.q[i]); }
            else { float lo, hi; norm::bf16x2_to_float(r0.q[i], lo, hi); v[2 * i] += lo; v[2 * i + 1] += hi; }
        }
    }
    if (YF) {
        float* p = static_cast<float*>(e.y) + y_off + col;
        Sector s;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s.q[i] = __float_as_uint(v[8 * h + i]);
            store_sector(p + 8 * h, s, e.wide_ok);
        }
    } else {
        store_sector(static_cast<__nv_bfloat16*>(e.y) + y_off + col, pack16(v), e.wide_ok);
    }
}

// Tile t of the launch: group_m row tiles are worked through column by column, so that what runs at one time shares rows of A
// and of B in L2.
__device__ __forceinline__ void tile_at(const TcArgs& a, int t, int& b, int& m, int& n) {
    const int all = a.batches * a.tiles_m, per_group = a.group_m * a.tiles_n;
    const int g = t / per_group, r = t - g * per_group, first = g * a.group_m, size = min(a.group_m, all - first);
    n = r / size;
    const int mt = first + r - n * size;
    b = mt / a.tiles_m;
    m = mt - b * a.tiles_m;
}

// Every CTA of the cluster finishes a run of the columns: the partial tiles of the same rows, added in the order of k.  By `step` threads from `from`, whole warps;
// the other warps of the cluster meet them at its barrier, ahead of which is worked out what does not depend on the shares.
__device__ __forceinline__ void join_shares(const TcArgs& a, uint32_t base, int first, uint32_t split, uint32_t half, const volatile int* abortp, int from, int step) {
    int b, m, n;
    tile_at(a, first, b, m, n);
    const uint32_t pitch = uint32_t(a.bn + 4) * 4u;
    const int share = a.bn / a.splits, groups = share / 8, c0 = int(split) * share;
    __syncwarp();
    cluster_sync();
    if (*abortp) return;
    for (int i = from; i < 128 * groups; i += step) {
        const int r = i / groups, c = c0 + (i - r * groups) * 8;
        const int row = m * kTileM + int(half) * 128 + r, col = n * a.bn + c, cn = min(max(a.cols - col, 0), 8);
        if (row >= a.rows || cn == 0) continue;
        norm::Raw8<true> res;
        if (a.e.residual) load_residual(a.e, b, row, col, cn, res);
        Columns cols;
        columns_begin(a.e, cols, col, cn);
        // all of the cluster's shares on their way before the first is added
        float g[4][8];
#pragma unroll
        for (int sp = 0; sp < 4; ++sp)
            if (sp < a.splits) {
                const uint32_t src = map_cta(base + uint32_t(r) * pitch + uint32_t(c) * 4u, uint32_t(2 * sp) + half);
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(g[sp][4 * q]), "=f"(g[sp][4 * q + 1]), "=f"(g[sp][4 * q + 2]),
                                 "=f"(g[sp][4 * q + 3]) : "r"(src + 16u * q) : "memory");
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) g[sp][q] = 0.f;
            }
        float f[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = ((g[0][q] + g[1][q]) + g[2][q]) + g[3][q];
        finish(a.e, cols, b, row, col, cn, f, res);
    }
}

constexpr int kLongRun = 2560;           // most k that one accumulator sums up for an fp32 output,
constexpr int kLongRunBf16 = 65536;      // and for a bf16 one

// kSub: slabs of 64 columns of k per stage.
// kLong: k is longer than one accumulator may sum up; 1: an fp32 output, a pair has all of k, 3: pairs share it, 2: a bf16 output, either.  The tensor cores cut
// their sums off instead of rounding them: a sum of 5120 products loses 5.6e-6 of itself, eight times what fp32 additions in a row do, and one of 524288 of the
// same sign (the rows of a weight's gradient) 3.8e-3, as much as the rounding to bf16; in runs 2.6e-5.  Here an accumulator sums up kRun
// stages of k at most, and the epilogue adds what it held to registers of its own, under the next run: 128 per thread, for which the service
// warps give most of theirs.  Pairs that share k do the same with their shares before they are joined (512 x 8960 x 2048 onto fp32, shares of 4480: 22.9 us,
// 21.8 in one run; 64 x 30720 x 1536, shares of 7680: 32.8 both ways, error 8.5e-6 in one run).  75600 x 5120 x 5120 onto a residual stream: error 1.6e-6
// with one run, 7.6e-7 with two, 2.8e-7 with five; 2848, 2903 and 3214 us.
template <int AMN, int BMN, int kSub, int kLong>
__global__ void __launch_bounds__(kThreadsTc, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapAs,
                 const __grid_constant__ CUtensorMap mapBs, const TcArgs a) {
    constexpr int kTileK = kSub * kSlab;                 // k of a stage
    constexpr uint32_t kABytes = 128 * kTileK * 2;       // a CTA's share of A per stage
    constexpr bool kF32 = kLong & 1, kShared = kLong != 1;               // pairs may share k
    constexpr int kRun = (kF32 ? kLongRun : kLongRunBf16) / kTileK;      // kLong: most stages of k that one accumulator sums up
    extern __shared__ unsigned char lin_smem[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(lin_smem) + 1023u) & ~1023u;
    const uint32_t bars = base + kRingBytes;
    const uint32_t rank = cluster_ctarank(), half = rank & 1u, leader = rank & ~1u, split = rank >> 1;
    const uint32_t b_bytes = uint32_t(a.bn / 2) * kTileK * 2, stage_bytes = kABytes + b_bytes;
    auto bar_full = [&](int s) { return bars + 8 * s; };                       // used in the pair's first CTA: both CTAs' copies have landed
    auto bar_empty = [&](int s) { return bars + 64 + 8 * s; };                 // the products that read stage s have completed
    auto bar_done = [&](int u) { return bars + 128 + 8 * u; };                 // accumulator u holds a tile
    auto bar_read = [&](int u) { return bars + 144 + 8 * u; };                 // first CTA: both CTAs have read accumulator u
    volatile int* abortp = &abort_flag;
    const unsigned long long limit = kDefaultWaitNs;
    const uint16_t pair_mask = uint16_t(3u << leader);

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < kMaxStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int u = 0; u < 2; ++u) { mbar_init(bar_done(u), 1); mbar_init(bar_read(u), 2 * kEpiWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 0 && lane == 0) {
        prefetch_tmap(&mapA); prefetch_tmap(&mapB);
        if (AMN) prefetch_tmap(&mapAs);
        if (BMN) prefetch_tmap(&mapBs);
    }
    grid_launch_dependents();
    tc_fence_before();
    __syncwarp();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    grid_wait();                         // launched while the kernel ahead drains: nothing of global memory is touched before this
    // the status word of the call: nothing sets it before its wait limit has passed, which is after this
    if (tid == 0 && blockIdx.x == 0 && a.clears) a.hdr->status = 0;
    __syncwarp();                        // whole warps hand over registers (setmaxnreg)

    // the clusters take the tiles in turn; with splits > 1 there is one cluster per tile and a pair has its share of k
    const int first = int(blockIdx.x / (2 * a.splits)), step = int(gridDim.x / (2 * a.splits));
    const int k_all = a.k_batches * a.k_tiles;
    const int k0 = int(int64_t(k_all) * split / a.splits), k1 = int(int64_t(k_all) * (split + 1) / a.splits);
    // kLong: runs of k with an accumulator each
    const int chunks = kLong ? (k1 - k0 + kRun - 1) / kRun : 1, chunk = (k1 - k0 + chunks - 1) / chunks;

    if (warp < 4) {                      // ---- service warps
    // 128 x 40 + 256 x 208 registers; the block is launched with 384 x 152 at least (checked by the host)
    if (kLong) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
    if (warp == 0) {
        // ================= TMA producer =================
        if (lane == 0) {
            const uint32_t full0 = map_cta(bar_full(0), leader);
            int s = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                int b, m, n;
                tile_at(a, t, b, m, n);
                const int m0 = m * kTileM + int(half) * 128, n0 = n * a.bn + int(half) * (a.bn / 2);
                int kb = k0 / a.k_tiles, kt = k0 - kb * a.k_tiles;
                for (int i = k0; i < k1; ++i) {
                    if (issued >= a.stages && !mbar_wait(bar_empty(s), phase ^ 1u, abortp, 0, limit)) {
                        set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 70, i, blockIdx.x); ok = false; break;
                    }
                    if (half == 0) mbar_expect_tx(bar_full(s), 2 * stage_bytes);
                    const uint32_t sa = base + uint32_t(s) * stage_bytes, sb = sa + kABytes, bar = full0 + 8 * s;
                    const int k = kt * kTileK;
                    if (AMN) {           // two slabs of 64 columns of m, the stage's rows of k
                        if (m0 / kSlab + 2 <= a.a_slabs) tma_load_pair_slabs(sa, &mapAs, bar, k, m0 / kSlab, kb);
                        else {
                            tma_load_pair(sa, &mapA, bar, m0, k, kb);
                            tma_load_pair(sa + kABytes / 2, &mapA, bar, m0 + kSlab, k, kb);
                        }
                    } else {             // slabs of 64 columns of k, 128 rows of m
                        for (int c = 0; c < kSub; ++c) tma_load_pair(sa + c * (kABytes / kSub), &mapA, bar, k + c * kSlab, m0, b);
                    }
                    if (BMN) {
                        if (n0 / kSlab + a.bn / 128 <= a.b_slabs) tma_load_pair_slabs(sb, &mapBs, bar, k, n0 / kSlab, kb);
                        else
                            for (int c = 0; c < a.bn / 2; c += kSlab) tma_load_pair(sb + uint32_t(c) * kTileK * 2, &mapB, bar, n0 + c, k, kb);
                    } else {
                        for (int c = 0; c < kSub; ++c) tma_load_pair(sb + uint32_t(c) * (b_bytes / kSub), &mapB, bar, k + c * kSlab, n0, 0);
                    }
                    ++issued;
                    if (++s == a.stages) { s = 0; phase ^= 1u; }
                    if (++kt == a.k_tiles) { kt = 0; ++kb; }
                }
            }
            // The completion of the last products on every stage: no copy is in flight and no arrival on its way to this CTA afterwards.
            const int used = min(issued, a.stages);
            for (int i = 0; i < used; ++i) {
                const int q = issued - used + i, sq = q % a.stages;
                const uint32_t par = uint32_t(q / a.stages) & 1u;
                if (*abortp ? !mbar_wait_drain(bar_empty(sq), par, 2000000ull) : !mbar_wait(bar_empty(sq), par, abortp, 0, limit))
                    set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 71, i, blockIdx.x);
            }
            if (*abortp) {               // given up: copies whose products were never issued land within microseconds
                const unsigned long long t0 = global_ns();
                for (int it = 0; it < 20000 && global_ns() - t0 < 1000000ull; ++it) __nanosleep(100);
            }
        }
    } else if (warp == 1) {
        // ================= MMA issuer (converged warp, one elected lane issues) =================
        if (half == 0) {
            const uint32_t idesc = instr_desc(kTileM, 0, BMN) | (uint32_t(a.bn >> 3) << 17) | (uint32_t(AMN) << 15);
            // K-major: 8-row groups 1024 B apart, 16 columns of k = 32 B, the next 64 in the next slab.  MN-major: 64-column slabs one behind the
            // other, 16 rows of k = 2 KB.
            const uint64_t da0 = AMN ? smem_desc(base, kABytes / 2, 1024) : smem_desc(base, 16, 1024);
            const uint64_t db0 = BMN ? smem_desc(base + kABytes, kTileK * 128, 1024) : smem_desc(base + kABytes, 16, 1024);
            const uint32_t a_lo = uint32_t(da0), a_hi = uint32_t(da0 >> 32), b_lo = uint32_t(db0), b_hi = uint32_t(db0 >> 32);
            const uint32_t slab_b = (b_bytes / kSub) >> 4;
            const int last = (a.k_len - (a.k_tiles - 1) * kTileK + 15) / 16;
            int s = 0, i = 0;
            uint32_t phase = 0;
            bool ok = true;
            int to_end = a.k_tiles - k0 % a.k_tiles;
            for (int c = 0, t = first; t < a.tiles && ok; ++i) {
                const int u = i & 1, from = k0 + c * chunk, to = min(from + chunk, k1);
                if (++c == chunks) { c = 0; t += step; }
                if (i >= 2) {
                    ok = mbar_wait_warp(bar_read(u), uint32_t((i >> 1) - 1) & 1u, abortp, 0, limit);
                    if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 72, i, blockIdx.x); break; }
                    tc_fence_after();
                }
                const uint32_t d = tmem + uint32_t(u) * 256u;
                for (int k = from; k < to; ++k) {
                    ok = mbar_wait_warp(bar_full(s), phase, abortp, 0, limit);
                    if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 73, k, blockIdx.x); break; }
                    tc_fence_after();
                    const uint32_t off = (uint32_t(s) * stage_bytes) >> 4;
                    auto product = [&](int kk) {
                        const uint32_t off_a = AMN ? kk * (2048 >> 4) : (kk / 4) * (kABytes / kSub >> 4) + (kk % 4) * 2;
                        const uint32_t off_b = BMN ? kk * (2048 >> 4) : (kk / 4) * slab_b + (kk % 4) * 2;
                        mma_pair_el(d, a_lo + off + off_a, a_hi, b_lo + off + off_b, b_hi, idesc, (k > from || kk > 0) ? 1u : 0u);
                    };
                    if (--to_end > 0) {
#pragma unroll
                        for (int kk = 0; kk < kTileK / 16; ++kk) product(kk);
                    } else {             // the end of a batch entry's k: what is all zero is left out
                        for (int kk = 0; kk < last; ++kk) product(kk);
                        to_end = a.k_tiles;
                    }
                    commit_pair_el(bar_empty(s), pair_mask);
                    if (++s == a.stages) { s = 0; phase ^= 1u; }
                }
                if (ok) commit_pair_el(bar_done(u), pair_mask);
            }
        }
    }
    if (kLong && kShared && a.splits > 1) {             // the epilogue warps meet the cluster before they join its tiles
        __syncwarp();
        cluster_sync();
    }
    } else {
        if (kLong) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;" ::: "memory");
        // ================= epilogue =================
        const int quarter = warp & 3, side = (warp - 4) >> 2;               // rows 32 quarter .. of this CTA's 128; every other 32 columns
        const uint32_t lane_base = uint32_t(quarter * 32) << 16;
        const uint32_t read0 = map_cta(bar_read(0), leader);
        bool ok = true;
        int i = 0;
        if (kLong) {
            for (int t = first; t < a.tiles && ok; t += step) {
                int b, m, n;
                tile_at(a, t, b, m, n);
                const int row = m * kTileM + int(half) * 128 + quarter * 32 + lane, left = min(a.cols - n * a.bn, a.bn);
                const bool on = row < a.rows;
                const int64_t y_off = b * a.e.ys[0] + row * a.e.ys[1], z_off = b * a.e.zs[0] + row * a.e.zs[1], r_off = b * a.e.rs[0] + row * a.e.rs[1];
                const int64_t gate_off = a.e.gate ? (b + row / a.e.rows_per_gate) * a.e.gate_stride : 0;
                const char* res = static_cast<const char*>(a.e.residual) + (r_off + n * a.bn) * (kF32 ? 4 : 2);
                __syncwarp();            // rows behind the last one have left the tile before early
                f2 acc[4][16];           // 32 columns each: side * 32, + 64, + 128, + 192
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int q = 0; q < 16; ++q) acc[p][q] = two(0.f);
                for (int c = 0; c < chunks && ok; ++c, ++i) {
                    const int u = i & 1;
                    ok = mbar_wait_warp(bar_done(u), uint32_t(i >> 1) & 1u, abortp, 20, limit);
                    if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 76, i, blockIdx.x); break; }
                    tc_fence_after();
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int at = side * 32 + 64 * p;
                        if (at < left) { // warp-uniform
                            float v[32];
                            tmem_ld32(tmem + lane_base + uint32_t(u * 256 + at), v);
                            tmem_wait_ld(v);
#pragma unroll
                            for (int q = 0; q < 16; ++q) acc[p][q] = add2(acc[p][q], two(v[2 * q], v[2 * q + 1]));
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_remote(read0 + 8 * u);
                }
                __syncwarp();
                if (!ok) break;
                if (kShared && a.splits > 1) {         // the one tile of this cluster: this pair's share to shared memory, as below
                    const uint32_t line = base + uint32_t(quarter * 32 + lane) * (uint32_t(a.bn + 4) * 4u);
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int at = side * 32 + 64 * p;
                        if (at < left) {
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                float f[4];
                                one_each(acc[p][2 * q], f[0], f[1]);
                                one_each(acc[p][2 * q + 1], f[2], f[3]);
                                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(line + uint32_t(at + 4 * q) * 4u), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
                            }
                        }
                    }
                    break;
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int at = side * 32 + 64 * p, col = n * a.bn + at;
                    if (at >= left || !on) continue;
                    if (at + 32 <= left) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            Sector r0, r1;
                            if (a.e.residual) {
                                r0 = load_sector(res + (at + 16 * h) * (kF32 ? 4 : 2), a.e.wide_ok);
                                if (kF32) r1 = load_sector(res + (at + 16 * h) * 4 + 32, a.e.wide_ok);
                            }
                            float f[16];
#pragma unroll
                            for (int q = 0; q < 8; ++q) one_each(acc[p][8 * h + q], f[2 * q], f[2 * q + 1]);
                            finish16<kF32>(a.e, a.e.gate, gate_off, y_off, z_off, col + 16 * h, f, r0, kF32 ? r1 : r0);
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const int cn = min(max(left - at - 8 * h, 0), 8);
                            if (cn > 0) {
                                norm::Raw8<true> r8;
                                Columns cols;
                                columns_begin(a.e, cols, col + 8 * h, cn);
                                if (a.e.residual) load_residual(a.e, b, row, col + 8 * h, cn, r8);
                                float f[8];
#pragma unroll
                                for (int q = 0; q < 4; ++q) one_each(acc[p][4 * h + q], f[2 * q], f[2 * q + 1]);
                                finish(a.e, cols, b, row, col + 8 * h, cn, f, r8);
                            }
                        }
                    }
                }
            }
            if (kShared && a.splits > 1) {
                tc_fence_before();
                join_shares(a, base, first, split, half, abortp, tid - 128, 32 * kEpiWarps);
            }
        } else if (a.splits == 1) {
            for (int t = first; t < a.tiles && ok; t += step, ++i) {
                const int u = i & 1;
                int b, m, n;
                tile_at(a, t, b, m, n);
                const int row = m * kTileM + int(half) * 128 + quarter * 32 + lane, left = min(a.cols - n * a.bn, a.bn);
                const bool on = row < a.rows;
                const int64_t y_off = b * a.e.ys[0] + row * a.e.ys[1], z_off = b * a.e.zs[0] + row * a.e.zs[1], r_off = b * a.e.rs[0] + row * a.e.rs[1];
                const int64_t gate_off = a.e.gate ? (b + row / a.e.rows_per_gate) * a.e.gate_stride : 0;
                const char* res = static_cast<const char*>(a.e.residual) + (r_off + n * a.bn) * (a.e.y_f32 ? 4 : 2);
                ok = mbar_wait_warp(bar_done(u), uint32_t(i >> 1) & 1u, abortp, 20, limit);
                if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 74, i, blockIdx.x); break; }
                tc_fence_after();
                for (int c = side * 32; c < left; c += 64) {               // warp-uniform
                    const int col = n * a.bn + c;
                    const bool whole = c + 32 <= left;
                    Sector r0, r1, r2, r3;
                    if (a.e.residual && whole && on) {
                        const char* p = res + c * (a.e.y_f32 ? 4 : 2);
                        r0 = load_sector(p, a.e.wide_ok); r1 = load_sector(p + 32, a.e.wide_ok);
                        if (a.e.y_f32) { r2 = load_sector(p + 64, a.e.wide_ok); r3 = load_sector(p + 96, a.e.wide_ok); }
                    }
                    __syncwarp();        // lanes of rows behind the last one have neither fetched this residual nor finished the columns before
                    float v[32];
                    tmem_ld32(tmem + lane_base + uint32_t(u * 256 + c), v);
                    tmem_wait_ld(v);
                    if (c + 64 >= left) {       // this warp has read its part of the tile
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_remote(read0 + 8 * u);
                    }
                    if (whole) {
                        float lo[16], hi[16];
#pragma unroll
                        for (int q = 0; q < 16; ++q) { lo[q] = v[q]; hi[q] = v[16 + q]; }
                        if (on && a.e.y_f32) {
                            finish16<true>(a.e, a.e.gate, gate_off, y_off, z_off, col, lo, r0, r1);
                            finish16<true>(a.e, a.e.gate, gate_off, y_off, z_off, col + 16, hi, r2, r3);
                        } else if (on) {
                            finish16<false>(a.e, a.e.gate, gate_off, y_off, z_off, col, lo, r0, r0);
                            finish16<false>(a.e, a.e.gate, gate_off, y_off, z_off, col + 16, hi, r1, r1);
                        }
                    } else if (on) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const int cn = min(max(left - c - 8 * h, 0), 8);
                            if (cn > 0) {
                                norm::Raw8<true> r8;
                                Columns cols;
                                columns_begin(a.e, cols, col + 8 * h, cn);
                                if (a.e.residual) load_residual(a.e, b, row, col + 8 * h, cn, r8);
                                float f[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q) f[q] = v[8 * h + q];
                                finish(a.e, cols, b, row, col + 8 * h, cn, f, r8);
                            }
                        }
                    }
                }
                if (side * 32 >= left) {
                    __syncwarp();
                    if (lane == 0) arrive_remote(read0 + 8 * u);
                }
            }
        } else {
            // partial tile to shared memory (every stage has been read by now: bar_done follows the last product)
            ok = mbar_wait_warp(bar_done(0), 0, abortp, 20, limit);
            if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 75, 0, blockIdx.x); }
            tc_fence_after();
            const uint32_t pitch = uint32_t(a.bn + 4) * 4u;
            if (ok)
                for (int c = side * 32; c < a.bn; c += 64) {
                    float v[32];
                    tmem_ld32(tmem + lane_base + uint32_t(c), v);
                    tmem_wait_ld(v);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(base + uint32_t(quarter * 32 + lane) * pitch + uint32_t(c + 4 * q) * 4u),
                                     "f"(v[4 * q]), "f"(v[4 * q + 1]), "f"(v[4 * q + 2]), "f"(v[4 * q + 3]) : "memory");
                }
            tc_fence_before();
        }
    }

    if (!kLong && a.splits > 1) join_shares(a, base, first, split, half, abortp, tid, kThreadsTc);
    tc_fence_before();
    __syncwarp();
    cluster_sync();                      // nothing of the cluster reads this CTA's memory or arrives on its barriers any more
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- host side ------------------------------------------------------------------------------------
// 3-D map over [batches, rows, cols] bf16 with the columns contiguous: box = 64 columns x box_rows x 1, 128-byte swizzle, what lies
// outside reads as zero.
inline bool make_map_3d(CUtensorMap* map, const void* base, int64_t batches, int64_t rows, int64_t cols, int64_t batch_stride, int64_t row_stride, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(batches)};
    // the stride of an axis of one entry is never used, but has to be a valid value
    const cuuint64_t row = rows > 1 ? cuuint64_t(row_stride) * 2 : cuuint64_t((cols + 7) / 8 * 16);
    cuuint64_t strides[2] = {row, batches > 1 ? cuuint64_t(batch_stride) * 2 : row};
    cuuint32_t box[3] = {64, cuuint32_t(box_rows), 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same for the whole slabs of 64 columns of an MN-major operand (the last one of another width would be read past the row): the columns as two dimensions, a box = 64 x box_rows x `slabs`, each
// slab landing as make_map_3d's box would.  One copy of 16 KB instead of two of 8: with two, dX and dW of 32760 x 1536 x 8960 took 637 and 650 us
// instead of 597 and 583.
inline bool make_map_slabs(CUtensorMap* map, const void* base, int64_t batches, int64_t rows, int64_t cols, int64_t batch_stride, int64_t row_stride, int box_rows,
                           int slabs) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {64, cuuint64_t(rows), cuuint64_t(cols / 64), cuuint64_t(batches)};
    const cuuint64_t row = rows > 1 ? cuuint64_t(row_stride) * 2 : cuuint64_t((cols + 7) / 8 * 16);
    cuuint64_t strides[3] = {row, 128, batches > 1 ? cuuint64_t(batch_stride) * 2 : row};
    cuuint32_t box[4] = {64, cuuint32_t(box_rows), cuuint32_t(slabs), 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A bf16 operand as [batches, rows, cols].
struct Operand { const void* base; int64_t batches, rows, cols, batch_stride, row_stride; };

// Columns of a tile and pairs that share one: the least time by a model in nanoseconds that was fitted to launches of 20 to 1000 rows.  A pair takes
// 75 + 0.85 columns per 64 of k (bounded by its products at 256 columns, by fetching its operands, 64 bytes a clock and SM, below), and an epilogue that is
// hidden except under very short k.  Joining two pairs costs 2.5 us, four 4.5 us (226 x 4096 x 1536: one pair per tile of 64 23.0 us, two per tile of 96
// 12.2, four per tile of 128 13.3; 64 x 9216 x 1536 20.3 with two, 15.4 with four).  33 clusters of 4 CTAs or 15 of 8 find room at a time; near
// that they start late.  Rows that start within a 64-byte piece (crooked) are fetched as more sectors: 1.6 times the time.
struct Plan { int bn, splits; };
inline Plan plan_of(int64_t m_tiles, int64_t cols, int64_t k_all, bool b_mn, bool crooked) {
    Plan best = {256, 1};
    double best_cost = 1e30;
    for (int bn = 256; bn >= (b_mn ? 128 : 64); bn -= b_mn ? 128 : 32) {
        const int64_t tiles = m_tiles * ((cols + bn - 1) / bn);
        for (int splits = 1; splits <= 4; splits *= 2) {
            if ((splits == 2 && tiles > 32) || (splits == 4 && tiles > 14) || k_all < 4 * splits * (splits > 1) || bn % (8 * splits)) break;
            const int64_t turns = splits > 1 ? 1 : (tiles + 73) / 74;
            const double k_ns = double((k_all + splits - 1) / splits) * (75 + 0.85 * bn) * (crooked ? 1.6 : 1.0), join = splits == 1 ? 0 : splits == 4 ? 4500 : tiles > 24 ? 4000 : 2500;
            const double cost = double(turns) * std::max(k_ns, 500.0 + 4 * bn) + join;
            if (cost < best_cost * 0.995) { best_cost = cost; best = {bn, splits}; }
        }
    }
    return best;
}

template <int AMN, int BMN, int kSub, int kLong>
inline carnator_status launch_tc_stages(const Operand& A, const Operand& B, TcArgs a, cudaStream_t stream, char* err, size_t errlen) {
    constexpr int kTileK = kSub * kSlab;
    const uint32_t stage = 128 * kTileK * 2 + uint32_t(a.bn / 2) * kTileK * 2;
    a.k_tiles = ceil_div(a.k_len, kTileK);
    a.stages = int(std::min<uint32_t>(kMaxStages, kRingBytes / stage));
    a.a_slabs = AMN ? int(A.cols / kSlab) : 0;
    a.b_slabs = BMN ? int(B.cols / kSlab) : 0;
    auto map = [](CUtensorMap* m, const Operand& o, int rows) { return make_map_3d(m, o.base, o.batches, o.rows, o.cols, o.batch_stride, o.row_stride, rows); };
    auto slabs = [](CUtensorMap* m, const CUtensorMap& plain, const Operand& o, int whole, int n) {
        if (whole > 0 && whole >= n) return make_map_slabs(m, o.base, o.batches, o.rows, o.cols, o.batch_stride, o.row_stride, kTileK, n);
        *m = plain;                      // not used
        return true;
    };
    CUtensorMap ma, mb, mas, mbs;
    if (!map(&ma, A, AMN ? kTileK : 128) || !map(&mb, B, BMN ? kTileK : a.bn / 2) || !slabs(&mas, ma, A, a.a_slabs, 2) || !slabs(&mbs, mb, B, a.b_slabs, a.bn / 128)) {
        snprintf(err, errlen, "cuTensorMapEncodeTiled failed or is unavailable");
        return CARNATOR_ERR_CUDA;
    }
    auto kern = linear_tc_kernel<AMN, BMN, kSub, kLong>;
    static SmemAllowed allowed;
    const unsigned long long ctx = context_id();
    if (!allowed.has(ctx)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemTc));
        if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(linear_tc_kernel)", err, errlen);
        if (kLong) {                     // the hand-over of registers only completes if the block owns them
            cudaFuncAttributes attr;
            const cudaError_t f = cudaFuncGetAttributes(&attr, kern);
            if (f != cudaSuccess) return cuda_error(f, "cudaFuncGetAttributes(linear_tc_kernel)", err, errlen);
            if (attr.numRegs * kThreadsTc < 128 * 40 + 256 * 208) {
                snprintf(err, errlen, "linear_tc_kernel was built with %d registers per thread: too few for its setmaxnreg split", attr.numRegs);
                return CARNATOR_ERR_UNSUPPORTED;
            }
        }
        allowed.add(ctx);
    }
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = unsigned(2 * a.splits); at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    const int clusters = a.splits > 1 ? a.tiles : std::min(a.tiles, 74);
    cfg.gridDim = dim3(unsigned(clusters * 2 * a.splits)); cfg.blockDim = dim3(kThreadsTc); cfg.dynamicSmemBytes = kSmemTc; cfg.stream = stream;
    cfg.attrs = at; cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ma, mb, mas, mbs, a);
    if (e != cudaSuccess) return cuda_error(e, "linear_tc_kernel", err, errlen);
    return CARNATOR_OK;
}

// The issuing warp spends about 200 clocks on a stage besides its products, which take it some 55 each, and a product of bn columns takes bn / 2: stages of 64 k
// keep up with 256 columns and leave the ring finer (32760 x 1536 x 8960 613 us, with 128 k 627 us), narrower tiles want stages of 128 k (512 x 4096
// x 5120 with 160 columns 23.5 and 19.5 us), as do MN-major operands, whose copies then are 32 KB each (dW of the former 627 and 615 us).
template <int AMN, int BMN>
inline carnator_status launch_tc_product(const Operand& A, const Operand& B, TcArgs a, cudaStream_t stream, char* err, size_t errlen) {
    const bool crooked = (A.rows > 1 && A.row_stride % 32) || (B.rows > 1 && B.row_stride % 32);
    const Plan p = plan_of(int64_t(a.batches) * a.tiles_m, a.cols, int64_t(a.k_batches) * ceil_div(a.k_len, kSlab), BMN, crooked);
    a.bn = p.bn; a.splits = p.splits;
    a.tiles_n = ceil_div(a.cols, a.bn);
    const int64_t tiles = int64_t(a.batches) * a.tiles_m * a.tiles_n;
    if (tiles > (int64_t(1) << 30)) return CARNATOR_ERR_UNSUPPORTED;
    a.tiles = int(tiles);
    a.group_m = 8;
    // whether a pair's share of k is longer than one accumulator may sum up
    const int64_t share = (int64_t(a.k_batches) * ceil_div(a.k_len, kSlab) + a.splits - 1) / a.splits;
    const bool longer = share * kSlab > (a.e.y_f32 ? kLongRun : kLongRunBf16);
    if constexpr (!AMN && !BMN) {
        if (longer && a.e.y_f32 && a.splits > 1)
            return a.bn == 256 ? launch_tc_stages<AMN, BMN, 1, 3>(A, B, a, stream, err, errlen) : launch_tc_stages<AMN, BMN, 2, 3>(A, B, a, stream, err, errlen);
        if (longer && a.e.y_f32) return a.bn == 256 ? launch_tc_stages<AMN, BMN, 1, 1>(A, B, a, stream, err, errlen) : launch_tc_stages<AMN, BMN, 2, 1>(A, B, a, stream, err, errlen);
        if (!longer && a.bn == 256) return launch_tc_stages<AMN, BMN, 1, 0>(A, B, a, stream, err, errlen);
    }
    return longer ? launch_tc_stages<AMN, BMN, 2, 2>(A, B, a, stream, err, errlen) : launch_tc_stages<AMN, BMN, 2, 0>(A, B, a, stream, err, errlen);
}

}  // namespace lin
}  // namespace carnator
