// Matrix product of 8-bit operands with a scale per block of 128 (fp8_quantize.cuh), on the 5th-gen tensor cores, with the epilogue of linear_tcgen05.cuh:
//   z = sum over blocks j of 128 k of  sx[row, j] sw[col / 128, j] <qx_j, qw_j>  + bias,   y = residual + gate_b act(z).
//
// Scales that are powers of two (fp8_quantize.cuh makes no others) are applied by the tensor cores: kind::mxf8f6f4 takes an exponent per row and 32 k from tensor memory
// (here the same for the four products of a block), so that an accumulator sums up all of k, or runs of 2560 of it for fp32 outputs.
// Any other scales: an accumulator sums up one block (kind::f8f6f4: products of two 4-bit significands are exact, a block's sum of them is cut off like any other; measured, all of
// k = 5120, 0.8 to 1.9 2^-24) and the epilogue warps take it times the block's scale into 128 fp32 sums per thread, while the next block's products run into the other
// accumulator.  That costs the reading and scaling of every block's sums, which bounds it: 9472 x 5120 x 5120 358 us against 205, and slower than the product in bf16.
// Otherwise bound by what an SM takes in (92 bytes a nanosecond) and, in long loops, by the power limit: 75600 x 5120 x 5120 in 1500 to 1770 us (1850 in a loop of a second at 1357 MHz and
// 990 W), onto an fp32 stream with a gate 1890 to 2030 (2370 at 1305 MHz).
// A first kernel quantises x where the call does, lays the exponents out as the tensor cores read them and notes whether all scales are powers of two; the product
// goes by its note, so that a caller does not have to say.
//
// A pair of CTAs shares a tile of 256 x BN (cta_group::2), as in linear_tcgen05.cuh, whose roles, ring and joining of shared sums these are.  BN <= 224: two accumulators
// and the exponents of four groups of four blocks fill tensor memory.
#pragma once
#include "fp8_quantize.cuh"
#include "linear_tcgen05.cuh"

namespace carnator {
namespace lin8 {
using namespace tc;
using namespace lin;
using fp8::kBlock;

constexpr uint32_t kABytes8 = 128 * kBlock;          // a CTA's share of A per stage
constexpr int kMostColumns = 224;                    // of a tile
constexpr int kGroupBlocks = 4;                      // blocks whose exponents share 32-bit words
constexpr uint32_t kSfA = 512, kSfB = 1024;          // bytes of a group's exponents: 128 rows, 256 columns
constexpr uint32_t kSfSlots = 10, kSfAt = 210 * 1024; // their ring in shared memory, behind the stages
constexpr uint32_t kSfColumn = 448;                  // first column of the exponents in tensor memory
static_assert(kSfAt + kSfSlots * (kSfA + kSfB) <= kRingBytes, "shared memory of a CTA");
enum { kXBf16 = 0, kXF32 = 1, kXE4m3 = 2 };

struct Args8 {
    TcArgs t;
    const float* xscale;                 // of an x that came in 8 bits, else NULL: its exponents are in sfa
    const float* wscale;
    const uint8_t* sfa;                  // [row tiles of 128][groups][512]
    const int* notes; int n_notes;       // not all zero: some scale is no power of two
    int64_t xss[3], wss[2];              // (batch, row, block), (block of columns, block)
    int groups;
};

// ---- the first kernel: x in 8 bits, exponents as tensor memory takes them -------------------------------------------------
// A group's exponents of 128 rows: a 32-bit word per row, byte j of it block 4 g + j; row r at 16 (r mod 32) + 4 (r / 32).
__device__ __forceinline__ int64_t sf_offset(int64_t tile, int groups, int g, int r) { return (tile * groups + g) * int64_t(kSfA) + (r & 31) * 16 + (r >> 5) * 4; }
// The exponent byte of a scale; what has none makes a note.  A NaN has one of its own.
__device__ __forceinline__ uint32_t exponent_of(float scale, int& note) {
    const uint32_t b = __float_as_uint(scale);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 255u;
    const uint32_t e = b >> 23;
    if ((b & 0x807FFFFFu) != 0u || e == 0u || e == 255u) { note = 1; return 127u; }
    return e;
}
struct PrepareArgs {
    fp8::QuantArgs q;                    // x (quantised here), or only rows, blocks, batches
    const float* xscale; const float* wscale;
    int64_t xss[3], wss[2];
    uint8_t* sfa; uint8_t* sfb;          // sfb: [column tiles][groups][1024], two times 128 columns
    int* notes;                          // one per CTA that looks at scales it was given
    WsHeader* hdr;
    int groups, row_tiles;               // row tiles of 128 per batch entry
    int cols, bn, tiles_n;
    int x_ctas, w_ctas;                  // CTAs per batch entry of x; behind all of them, those of the weight's scales
};
template <int kType>
__global__ void __launch_bounds__(fp8::kRowThreads, 4) prepare_fp8_kernel(const PrepareArgs a) {
    const int x_all = a.x_ctas * a.q.batches, tid = threadIdx.x;
    const bool of_x = int(blockIdx.x) < x_all;
    const int b = of_x ? int(blockIdx.x) / a.x_ctas : 0, cta = int(blockIdx.x) - (of_x ? b * a.x_ctas : x_all);
    grid_launch_dependents();
    grid_wait();
    if (blockIdx.x == 0 && tid == 0) a.hdr->status = 0;
    int note = 0;
    if (of_x) {
        if constexpr (kType == kXE4m3) {
            const int64_t items = int64_t(a.groups) * a.q.rows;
            for (int64_t i = int64_t(cta) * fp8::kRowThreads + tid; i < items; i += int64_t(a.x_ctas) * fp8::kRowThreads) {
                const int g = int(i / a.q.rows), row = int(i - int64_t(g) * a.q.rows);
                const float* p = a.xscale + b * a.xss[0] + row * a.xss[1];
                uint32_t word = 0;
#pragma unroll
                for (int j = 0; j < kGroupBlocks; ++j)
                    if (g * kGroupBlocks + j < a.q.blocks) word |= exponent_of(p[(g * kGroupBlocks + j) * a.xss[2]], note) << (8 * j);
                *reinterpret_cast<uint32_t*>(a.sfa + sf_offset(int64_t(b) * a.row_tiles + row / 128, a.groups, g, row % 128)) = word;
            }
        } else {
            constexpr bool kF = kType == kXF32;
            constexpr int kAhead = fp8::kAheadOf<kF>;
            static_assert(kGroupBlocks % kAhead == 0, "a lane's blocks lie within a word");
            fp8::quantize_rows<kF, kAhead>(a.q, b, cta, a.x_ctas, [&](int row, int blk, const float (&scale)[kAhead]) {
                int none = 0;
                uint32_t word = 0;
#pragma unroll
                for (int k = 0; k < kAhead; ++k) word |= exponent_of(scale[k], none) << (8 * k);
                uint8_t* to = a.sfa + sf_offset(int64_t(b) * a.row_tiles + row / 128, a.groups, blk / kGroupBlocks, row % 128) + blk % kGroupBlocks;
                if (kAhead == 4) *reinterpret_cast<uint32_t*>(to) = word;
                else *reinterpret_cast<uint16_t*>(to) = uint16_t(word);
            });
        }
    } else {
        const int64_t words = int64_t(a.tiles_n) * a.groups * 256;
        for (int64_t i = int64_t(cta) * fp8::kRowThreads + tid; i < words; i += int64_t(a.w_ctas) * fp8::kRowThreads) {
            const int c = int(i & 255);
            const int64_t tg = i >> 8;
            const int n = int(tg / a.groups), g = int(tg - int64_t(n) * a.groups), col = n * a.bn + c;
            uint32_t word = 0x7F7F7F7Fu;
            if (c < a.bn && col < a.cols) {
                const float* p = a.wscale + (col / kBlock) * a.wss[0];
                word = 0;
#pragma unroll
                for (int j = 0; j < kGroupBlocks; ++j)
                    if (g * kGroupBlocks + j < a.q.blocks) word |= exponent_of(p[(g * kGroupBlocks + j) * a.wss[1]], note) << (8 * j);
            }
            *reinterpret_cast<uint32_t*>(a.sfb + tg * kSfB + (c >> 7) * 512 + (c & 31) * 16 + ((c & 127) >> 5) * 4) = word;
        }
    }
    if (of_x && kType != kXE4m3) return; // x that is quantised here has powers of two
    note = __syncthreads_or(note);
    if (tid == 0) a.notes[of_x ? a.w_ctas + int(blockIdx.x) : cta] = note;
}

// ---- the product ------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma8_pair_el(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], da, db, %5, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// the same with an exponent per row of either operand, byte `id` (in the descriptor) of the words at these columns
__device__ __forceinline__ void mma8_scaled_pair_el(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t sa, uint32_t sb,
                                                    uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %8, 0;\n\t"
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], da, db, %5, [%6], [%7], p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
// 512 bytes of shared memory (of both CTAs) into four columns, the same for each of the four quarters of the lanes
__device__ __forceinline__ void copy_exponents_el(uint32_t tmem, uint32_t smem) {
    // no swizzle: 8 rows of 16 bytes beside each other, the next 8 rows 128 bytes on
    const uint64_t desc = uint64_t((smem & 0x3FFFFu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
        ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ float load_scale(const float* p) {      // not through the read-only path: the kernel ahead may write it while this one is resident
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float scale_from(uint32_t word, int j) {
    const uint32_t e = (word >> (8 * j)) & 255u;
    return __uint_as_float(e == 255u ? 0x7FC00000u : e << 23);
}

// What an epilogue warp is told.
struct Epi {
    uint32_t tmem, base, bars, read0;    // read0: the first of the barriers on which accumulators are given back, in the pair's first CTA
    int half, first, step, k0, k1, chunks;
    volatile int* abortp;
};
enum { kAtOnce, kEachRun, kEachBlock };  // an accumulator holds a tile's whole sum, a run of it, or that of one block without its scales
// Its tiles; a shared one is left in shared memory.  (Three functions, so that what one way holds in registers does not cost another: in one loop, the sums of the
// third spilled 3 KB, what the first needs among it: 75600 x 5120 x 5120 onto an fp32 stream 2889 us, apart 1830.  What is left, where sums are held beside a tile's end: 266 bytes of
// stores and 300 of loads in the fp32 kernels, 120 and 104 in the bf16 ones.)
template <bool kF32, int kMode>
__device__ __forceinline__ void epilogue_warp(const Args8& args, const Epi& c) {
    const TcArgs& a = args.t;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quarter = warp & 3, side = (warp - 4) >> 2;               // rows 32 quarter .. of this CTA's 128; every other 32 columns
    const uint32_t tmem = c.tmem + (uint32_t(quarter * 32) << 16);
    const uint32_t line = c.base + uint32_t(quarter * 32 + lane) * (uint32_t(a.bn + 4) * 4u);        // of a shared tile
    bool ok = true;
    int i = 0, s = 0;
    uint32_t phase = 0;
    auto release = [&](int u) __attribute__((always_inline)) {      // this warp has read its part of accumulator u
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_remote(c.read0 + 8 * u);
    };
    for (int t = c.first; t < a.tiles && ok; t += c.step) {
        int b, m, n;
        tile_at(a, t, b, m, n);
        const int row = m * kTileM + c.half * 128 + quarter * 32 + lane, left = min(a.cols - n * a.bn, a.bn);
        const bool on = row < a.rows;
        struct Where { int64_t y, gate; const char* res; };          // of this row, worked out where the tile ends: registers are short before that
        auto where = [&]() __attribute__((always_inline)) {
            Where w;
            w.y = b * a.e.ys[0] + row * a.e.ys[1];
            w.gate = a.e.gate ? (b + row / a.e.rows_per_gate) * a.e.gate_stride : 0;
            w.res = static_cast<const char*>(a.e.residual) + (b * a.e.rs[0] + row * a.e.rs[1] + n * a.bn) * (kF32 ? 4 : 2);
            return w;
        };
        // A tile ends in steps of 16 columns.  `r`: their residual, where all of them are there.
        auto fetch = [&](const Where& w, int at, Sector (&r)[kF32 ? 2 : 1]) __attribute__((always_inline)) {
            if (a.e.residual && a.splits == 1 && on && at + 16 <= left) {
#pragma unroll
                for (int h = 0; h < (kF32 ? 2 : 1); ++h) r[h] = load_sector(w.res + at * (kF32 ? 4 : 2) + 32 * h, a.e.wide_ok);
            }
        };
        auto end_of = [&](const Where& w, int at, float (&f)[16], const Sector (&r)[kF32 ? 2 : 1]) __attribute__((always_inline)) {
            const int col = n * a.bn + at;
            if (a.splits > 1) {          // the one tile of this cluster: this pair's share to shared memory
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(line + uint32_t(at + 4 * q) * 4u), "f"(f[4 * q]), "f"(f[4 * q + 1]), "f"(f[4 * q + 2]), "f"(f[4 * q + 3]) : "memory");
            } else if (at + 16 <= left) {
                if (on) finish16<kF32>(a.e, a.e.gate, w.gate, w.y, 0, col, f, r[0], r[kF32 ? 1 : 0]);
            } else if (on) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int cn = min(max(left - at - 8 * h, 0), 8);
                    if (cn > 0) {
                        norm::Raw8<true> r8;
                        Columns cols;
                        columns_begin(a.e, cols, col + 8 * h, cn);
                        if (a.e.residual) load_residual(a.e, b, row, col + 8 * h, cn, r8);
                        float g[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) g[q] = f[8 * h + q];
                        finish(a.e, cols, b, row, col + 8 * h, cn, g, r8);
                    }
                }
            }
        };
        __syncwarp();                // rows behind the last one have left the tile before early
        if constexpr (kMode == kAtOnce) {
            const int u = i & 1;
            // this step's residual, the next one's and the one's behind it, of which the first two are fetched under the products
            Sector r0[kF32 ? 2 : 1], r1[kF32 ? 2 : 1], r2[kF32 ? 2 : 1];
            auto column = [&](int st) { return side * 32 + 64 * (st >> 1) + 16 * (st & 1); };
            const Where w = where();
            fetch(w, column(0), r0);
            fetch(w, column(1), r1);
            ok = mbar_wait_warp(c.bars + 128 + 8 * u, uint32_t(i >> 1) & 1u, c.abortp, 20, kDefaultWaitNs);
            if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 84, i, blockIdx.x); break; }
            tc_fence_after();
            ++i;
            // `next` is filled for the step after the next: three in turn, so that none is moved while it is on its way
            auto step_of = [&](int st, const Sector (&mine)[kF32 ? 2 : 1], Sector (&next)[kF32 ? 2 : 1]) __attribute__((always_inline)) {
                if (column(st) >= left) return;      // warp-uniform
                float v[16];
                __syncwarp();            // lanes of rows behind the last one have not finished the columns before
                tmem_ld16(tmem + uint32_t(u * kMostColumns + column(st)), v);
                fetch(w, column(st + 2), next);
                __syncwarp();
                tmem_wait_ld(v);
                if (column(st + 1) >= left) release(u);
                end_of(w, column(st), v, mine);
            };
#pragma unroll 1
            for (int st = 0; column(st) < left; st += 3) {
                step_of(st, r0, r2);
                step_of(st + 1, r1, r0);
                step_of(st + 2, r2, r1);
            }
            if (side * 32 >= left) release(u);
            if (a.splits > 1) break;
        } else {
        f2 acc[4][16];               // 32 columns each: side * 32, + 64, + 128, + 192
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[p][q] = two(0.f);
        if constexpr (kMode == kEachRun) {
            for (int r = 0; r < c.chunks && ok; ++r, ++i) {
                const int u = i & 1;
                ok = mbar_wait_warp(c.bars + 128 + 8 * u, uint32_t(i >> 1) & 1u, c.abortp, 20, kDefaultWaitNs);
                if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 85, i, blockIdx.x); break; }
                tc_fence_after();
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int at = side * 32 + 64 * p;
                    if (at < left) {
                        float v[32];
                        tmem_ld32(tmem + uint32_t(u * kMostColumns + at), v);
                        tmem_wait_ld(v);
#pragma unroll
                        for (int q = 0; q < 16; ++q) acc[p][q] = norm::add2(acc[p][q], two(v[2 * q], v[2 * q + 1]));
                    }
                }
                release(u);
            }
        } else {
            // x's scales of four blocks are on their way while the four before are used (one block ahead, every block waited for them); the weight's of 32 blocks, one per
            // lane, for each 32 columns
            const float* xs = args.xscale ? args.xscale + b * args.xss[0] + (on ? row : 0) * args.xss[1] : nullptr;
            const uint8_t* xe = args.sfa + sf_offset((int64_t(b) * a.tiles_m + m) * 2 + c.half, args.groups, 0, quarter * 32 + lane);
            float wv[4], xn[4];
            auto scales = [&](int g) __attribute__((always_inline)) {
                if (xs) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) xn[j] = load_scale(xs + min(g + j, c.k1 - 1) * args.xss[2]);
                } else {
                    const uint32_t word = __float_as_uint(load_scale(reinterpret_cast<const float*>(xe + int64_t(min(g, c.k1 - 1) / kGroupBlocks) * kSfA)));
#pragma unroll
                    for (int j = 0; j < 4; ++j) xn[j] = scale_from(word, j);
                }
            };
            scales(c.k0);
            for (int g = c.k0; g < c.k1 && ok; g += 4) {
                float xv[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) xv[j] = xn[j];
                if (((g - c.k0) & 31) == 0) {
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        wv[p] = load_scale(args.wscale + (min(n * a.bn + side * 32 + 64 * p, a.cols - 1) / kBlock) * args.wss[0] + min(g + lane, c.k1 - 1) * args.wss[1]);
                }
                scales(g + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int k = g + j, u = i & 1;
                    if (k >= c.k1) break;
                    ok = mbar_wait_warp(c.bars + 64 + 8 * s, phase, c.abortp, 0, kDefaultWaitNs);
                    if (!ok) { if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 86, i, blockIdx.x); break; }
                    ++i;
                    if (++s == a.stages) { s = 0; phase ^= 1u; }
                    tc_fence_after();
                    const uint32_t from = tmem + uint32_t(u * kMostColumns + side * 32);
                    // All four pieces of 32 columns, whether the tile has them or not: what it has not is added to sums that nobody reads.  (9472 x 5120 x 5120, us: as here
                    // 358, with a branch around each piece 447, pieces of 16 in turn, one on its way while the other is added, 420 and, with branches, 422)
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const f2 by = two(xv[j] * __shfl_sync(0xffffffffu, wv[p], (k - c.k0) & 31));
                        float v[32];
                        tmem_ld32(from + 64 * p, v);
                        tmem_wait_ld(v);
#pragma unroll
                        for (int q = 0; q < 16; ++q) acc[p][q] = norm::fma2(two(v[2 * q], v[2 * q + 1]), by, acc[p][q]);
                    }
                    release(u);
                }
            }
        }
        __syncwarp();
        if (!ok) break;
        const Where w = where();
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = side * 32 + 64 * p + 16 * h;
                if (at < left) {     // warp-uniform
                    Sector r[kF32 ? 2 : 1];
                    fetch(w, at, r);
                    float v[16];
#pragma unroll
                    for (int q = 0; q < 8; ++q) one_each(acc[p][8 * h + q], v[2 * q], v[2 * q + 1]);
                    end_of(w, at, v, r);
                }
            }
        if (a.splits > 1) break;     // the one tile of this cluster
        }
    }
}

// kRuns: an accumulator sums up runs of k only, which the epilogue adds in registers (longer sums than one may take up).
template <bool kF32, bool kRuns>
__global__ void __launch_bounds__(kThreadsTc, 1)
linear_fp8_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapSa,
                  const __grid_constant__ CUtensorMap mapSb, const Args8 args) {
    // Most k that one accumulator sums up, as in linear_tcgen05.cuh: the tensor cores cut their sums off (measured, quantised normal values: error of a sum of 2560 1.7e-7, of
    // 5120 3.6e-7, of 10240 8.5e-7; all terms positive 7.0e-7, 2.0e-6, 5.2e-6; with scales 16-fold apart, runs of 2560 1.2e-6, of 5120 2.9e-6).  Runs of 5120 for fp32 outputs took 1849 us instead of 1893 at 75600 x 5120 x 5120 with gate and residual,
    // 24.5 instead of 25.6 at 512 x 4096 x 5120.
    constexpr int kRun = (kF32 ? kLongRun : kLongRunBf16) / kBlock;
    static_assert(kRun % kGroupBlocks == 0, "runs are whole groups");
    const TcArgs& a = args.t;
    extern __shared__ unsigned char lin_smem[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(lin_smem) + 1023u) & ~1023u;
    const uint32_t bars = base + kRingBytes;
    const uint32_t rank = cluster_ctarank(), half = rank & 1u, leader = rank & ~1u, split = rank >> 1;
    const uint32_t stage_bytes = kABytes8 + uint32_t(a.bn / 2) * kBlock;
    auto bar_full = [&](int s) { return bars + 8 * s; };                       // used in the pair's first CTA: both CTAs' copies have landed
    auto bar_done = [&](int s) { return bars + 64 + 8 * s; };                  // the products of stage s have completed
    auto bar_sum = [&](int u) { return bars + 128 + 8 * u; };                  // accumulator u holds a run
    auto bar_read = [&](int u) { return bars + 144 + 8 * u; };                 // first CTA: both CTAs have read accumulator u
    volatile int* abortp = &abort_flag;
    const unsigned long long limit = kDefaultWaitNs;
    const uint16_t pair_mask = uint16_t(3u << leader);

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < kMaxStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_done(s), 1); }
        for (int u = 0; u < 2; ++u) { mbar_init(bar_sum(u), 1); mbar_init(bar_read(u), 2 * kEpiWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 0 && lane == 0) { prefetch_tmap(&mapA); prefetch_tmap(&mapB); prefetch_tmap(&mapSa); prefetch_tmap(&mapSb); }
    grid_launch_dependents();
    tc_fence_before();
    __syncwarp();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    grid_wait();                         // launched while the kernel ahead drains: nothing of global memory is touched before this
    // Whether all of the call's scales are powers of two: the same in every CTA.  Each warp looks for itself, while the first copies are on their way.
    auto all_powers = [&]() {
        int note = 0;
#pragma unroll 4
        for (int i = lane; i < args.n_notes; i += 32) note |= reinterpret_cast<const volatile int*>(args.notes)[i];
        return __any_sync(0xffffffffu, note != 0) == 0;
    };
    __syncwarp();                        // whole warps hand over registers (setmaxnreg)

    // the clusters take the tiles in turn; with splits > 1 there is one cluster per tile and a pair has its share of k, in whole groups
    const int first = int(blockIdx.x / (2 * a.splits)), step = int(gridDim.x / (2 * a.splits));
    const int k0 = int(int64_t(args.groups) * split / a.splits) * kGroupBlocks, k1 = min(int(int64_t(args.groups) * (split + 1) / a.splits) * kGroupBlocks, a.k_tiles);
    // runs of k with an accumulator each
    const int chunks = kRuns ? (k1 - k0 + kRun - 1) / kRun : 1, chunk = kRuns ? kRun : k1 - k0;

    if (warp < 4) {                      // ---- service warps
    // 128 x 40 + 256 x 208 registers; the block is launched with 384 x 152 at least (checked by the host)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
    if (warp == 0) {
        // ================= TMA producer =================
        if (lane == 0) {
            const uint32_t full0 = map_cta(bar_full(0), leader);
            int s = 0, issued = 0, group = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                int b, m, n;
                tile_at(a, t, b, m, n);
                const int m0 = m * kTileM + int(half) * 128, n0 = n * a.bn + int(half) * (a.bn / 2);
                const int sf_row = ((b * a.tiles_m + m) * 2 + int(half)) * args.groups, sf_col = n * args.groups;
                for (int k = k0; k < k1; ++k) {
                    if (issued >= a.stages && !mbar_wait(bar_done(s), phase ^ 1u, abortp, 0, limit)) {
                        set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 80, k, blockIdx.x); ok = false; break;
                    }
                    const bool sf = k % kGroupBlocks == 0;             // used or not
                    if (half == 0) mbar_expect_tx(bar_full(s), 2 * (stage_bytes + (sf ? kSfA + kSfB : 0u)));
                    const uint32_t sa = base + uint32_t(s) * stage_bytes, bar = full0 + 8 * s;
                    if (sf) {            // its slot: of the group kSfSlots back, whose last block lies further back than there are stages
                        const uint32_t to = base + kSfAt + uint32_t(group % int(kSfSlots)) * (kSfA + kSfB);
                        tma_load_pair(to, &mapSa, bar, 0, sf_row + k / kGroupBlocks, 0);
                        tma_load_pair(to + kSfA, &mapSb, bar, 0, sf_col + k / kGroupBlocks, 0);
                        ++group;
                    }
                    tma_load_pair(sa, &mapA, bar, k * kBlock, m0, b);
                    tma_load_pair(sa + kABytes8, &mapB, bar, k * kBlock, n0, 0);
                    ++issued;
                    if (++s == a.stages) { s = 0; phase ^= 1u; }
                }
            }
            // The completion of the last products on every stage: no copy is in flight and no arrival on its way to this CTA afterwards.
            const int used = min(issued, a.stages);
            for (int i = 0; i < used; ++i) {
                const int q = issued - used + i, sq = q % a.stages;
                const uint32_t par = uint32_t(q / a.stages) & 1u;
                if (*abortp ? !mbar_wait_drain(bar_done(sq), par, 2000000ull) : !mbar_wait(bar_done(sq), par, abortp, 0, limit))
                    set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 81, i, blockIdx.x);
            }
            if (*abortp) {               // given up: copies whose products were never issued land within microseconds
                const unsigned long long t0 = global_ns();
                for (int it = 0; it < 20000 && global_ns() - t0 < 1000000ull; ++it) __nanosleep(100);
            }
        }
    } else if (warp == 1) {
        // ================= MMA issuer (converged warp, one elected lane issues) =================
        if (half == 0) {
            // e4m3 x e4m3, fp32 accumulator; K-major operands: 8-row groups 1024 B apart, 32 columns of k = 32 B
            const uint32_t idesc = (1u << 4) | (uint32_t(a.bn >> 3) << 17) | (uint32_t(kTileM >> 4) << 24);
            const uint32_t idesc_sf = (1u << 23) | (uint32_t(a.bn >> 3) << 17) | (uint32_t(kTileM >> 7) << 27);      // exponents as scales
            const uint64_t da0 = smem_desc(base, 16, 1024), db0 = smem_desc(base + kABytes8, 16, 1024);
            const uint32_t a_lo = uint32_t(da0), a_hi = uint32_t(da0 >> 32), b_lo = uint32_t(db0), b_hi = uint32_t(db0 >> 32);
            const int last = (a.k_len - (a.k_tiles - 1) * kBlock + 31) / 32;
            const bool scaled = all_powers();
            int s = 0, i = 0, group = 0;
            uint32_t phase = 0;
            bool ok = true;
            auto free_accumulator = [&](int u) {
                if (i < 2) return true;
                if (mbar_wait_warp(bar_read(u), uint32_t((i >> 1) - 1) & 1u, abortp, 0, limit)) return true;
                if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 82, i, blockIdx.x);
                return false;
            };
            auto full_stage = [&](int k) {
                if (mbar_wait_warp(bar_full(s), phase, abortp, 0, limit)) return true;
                if (lane == 0) set_status(a.hdr, CARNATOR_ERR_DEVICE_TIMEOUT, 83, k, blockIdx.x);
                return false;
            };
            for (int t = first; t < a.tiles && ok; t += step) {
                if (scaled) {
                    for (int c = 0; c < chunks && ok; ++c, ++i) {
                        const int u = i & 1, from = k0 + c * chunk, to = min(from + chunk, k1);
                        if (!(ok = free_accumulator(u))) break;
                        const uint32_t d = tmem + uint32_t(u * kMostColumns);
                        uint32_t sf = 0;
                        for (int k = from; k < to; ++k) {
                            if (!(ok = full_stage(k))) break;
                            tc_fence_after();
                            if (k % kGroupBlocks == 0) {
                                const uint32_t at = base + kSfAt + uint32_t(group % int(kSfSlots)) * (kSfA + kSfB);
                                sf = tmem + kSfColumn + uint32_t(group & 3) * 16u;
                                copy_exponents_el(sf, at);
                                copy_exponents_el(sf + 4, at + kSfA);
                                copy_exponents_el(sf + 8, at + kSfA + 512);
                                ++group;
                            }
                            const uint32_t off = (uint32_t(s) * stage_bytes) >> 4, id = uint32_t(k % kGroupBlocks), ids = idesc_sf | id << 4 | id << 29;
                            if (k + 1 < a.k_tiles) {
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk)
                                    mma8_scaled_pair_el(d, a_lo + off + kk * 2, a_hi, b_lo + off + kk * 2, b_hi, ids, sf, sf + 4, k > from || kk > 0 ? 1u : 0u);
                            } else {     // the end of k: what is all zero is left out
                                for (int kk = 0; kk < last; ++kk)
                                    mma8_scaled_pair_el(d, a_lo + off + kk * 2, a_hi, b_lo + off + kk * 2, b_hi, ids, sf, sf + 4, k > from || kk > 0 ? 1u : 0u);
                            }
                            commit_pair_el(bar_done(s), pair_mask);
                            if (++s == a.stages) { s = 0; phase ^= 1u; }
                        }
                        if (ok) commit_pair_el(bar_sum(u), pair_mask);
                    }
                } else {
                    for (int k = k0; k < k1 && ok; ++k, ++i) {
                        const int u = i & 1;
                        if (!(ok = free_accumulator(u)) || !(ok = full_stage(k))) break;
                        tc_fence_after();
                        const uint32_t off = (uint32_t(s) * stage_bytes) >> 4, d = tmem + uint32_t(u * kMostColumns);
                        const int n = k + 1 < a.k_tiles ? 4 : last;
                        for (int kk = 0; kk < n; ++kk) mma8_pair_el(d, a_lo + off + kk * 2, a_hi, b_lo + off + kk * 2, b_hi, idesc, kk > 0 ? 1u : 0u);
                        commit_pair_el(bar_done(s), pair_mask);
                        if (++s == a.stages) { s = 0; phase ^= 1u; }
                    }
                }
            }
        }
    }
    if (a.splits > 1) {                  // the epilogue warps meet the cluster before they join its tiles
        __syncwarp();
        cluster_sync();
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;" ::: "memory");
        // ================= epilogue =================
        const Epi c = {tmem, base, bars, map_cta(bars + 144, leader), int(half), first, step, k0, k1, chunks, abortp};
        if (!all_powers()) epilogue_warp<kF32, kEachBlock>(args, c);
        else epilogue_warp<kF32, kRuns ? kEachRun : kAtOnce>(args, c);
        if (a.splits > 1) {
            tc_fence_before();
            join_shares(a, base, first, split, half, abortp, tid - 128, 32 * kEpiWarps);
        }
    }

    tc_fence_before();
    __syncwarp();
    cluster_sync();                      // nothing of the cluster reads this CTA's memory or arrives on its barriers any more
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- a few rows ---------------------------------------------------------------------------------------
// All that a few rows have to move is W, once: as in linear_rows.cuh a CTA takes 16 rows of W, its warps share k (here in blocks of 128), and lanes fetch W
// straight into the registers of mma.m16n8k32.  x is taken to 8 bits by every CTA for itself, in the registers of the same instruction: a lane has 2 x 16 channels
// of a block of one row, four lanes the block.  One launch.
constexpr int kRowsMost8 = 16;
struct RowsArgs8 {
    Epilogue e;
    const void* x; const uint8_t* w;
    const float* xscale; const float* wscale;
    int64_t xs[2], xss[3], w_stride, wss[2];
    WsHeader* hdr;
    int rows, per_batch, K, cols;        // rows over all batch entries; rows of an entry
};

__device__ __forceinline__ uint4 load_q16(const uint8_t* row, int k, int K) {
    if (k + 16 <= K) {
        uint4 v;
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + k));
        return v;
    }
    uint32_t t[4] = {0, 0, 0, 0};        // the last k of a row: what lies behind them is not the row's
    if (k >= K) return make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k + i < K) t[i / 4] |= uint32_t(*reinterpret_cast<const volatile uint8_t*>(row + k + i)) << (8 * (i & 3));
    return make_uint4(t[0], t[1], t[2], t[3]);
}
__device__ __forceinline__ void mma_16x8x32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT: column tiles of 8 rows of x; kWarps: warps that share k; kType: of x; FT: tiles of 16 rows of W, which share x in 8 bits
template <int NT, int kWarps, int kType, int FT>
__global__ void __launch_bounds__(32 * kWarps) linear_fp8_rows_kernel(const RowsArgs8 a) {
    __shared__ float sums[kWarps][16 * FT][8 * NT + 1];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    grid_launch_dependents();
    grid_wait();                         // launched while the kernel ahead drains
    if (blockIdx.x == 0 && tid == 0) a.hdr->status = 0;
    const int f0 = blockIdx.x * 16 * FT, blocks = (a.K + kBlock - 1) / kBlock;
    const uint8_t* w0 = a.w + int64_t(f0 + g) * a.w_stride;
    const float* ws = a.wscale + (f0 / kBlock) * a.wss[0];       // 16 FT divides a block
    int64_t xo[NT], so[NT];
    bool xon[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int row = j * 8 + g;
        xon[j] = row < a.rows;
        const int b = xon[j] ? row / a.per_batch : 0, r = xon[j] ? row - b * a.per_batch : 0;
        xo[j] = b * a.xs[0] + r * a.xs[1];
        so[j] = b * a.xss[0] + r * a.xss[1];
    }
    float acc[FT][NT][4];
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[f][j][i] = 0.f;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    constexpr int U = NT == 1 && FT <= 2 ? 2 : 1;    // blocks in flight per warp
    for (int blk = warp; blk < blocks; blk += kWarps * U) {
        uint4 u[U][FT][2][2];            // of rows g and g + 8 of each tile, two pieces of k
        float sw[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const int kb = blk + q * kWarps;         // past the end: zeros
#pragma unroll
            for (int f = 0; f < FT; ++f)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const bool on = f0 + 16 * f + 8 * r + g < a.cols;
#pragma unroll
                    for (int h = 0; h < 2; ++h) u[q][f][r][h] = on ? load_q16(w0 + (16 * f + 8 * r) * a.w_stride, kb * kBlock + h * 64 + t * 16, a.K) : zero;
                }
            sw[q] = kb < blocks ? load_scale(ws + kb * a.wss[1]) : 0.f;
        }
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const int kb = blk + q * kWarps;
            if (kb >= blocks) break;     // warp-uniform
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint4 xq[2];
                float sx;
                if constexpr (kType == kXE4m3) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) xq[h] = xon[j] ? load_q16(static_cast<const uint8_t*>(a.x) + xo[j], kb * kBlock + h * 64 + t * 16, a.K) : zero;
                    sx = xon[j] ? load_scale(a.xscale + so[j] + kb * a.xss[2]) : 0.f;
                } else {
                    fp8::Lane16<kType == kXF32> v[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = kb * kBlock + h * 64 + t * 16;
                        v[h].load(a.x, xo[j] + k, xon[j] ? a.K - k : 0);
                    }
                    uint32_t m = max(v[0].most(), v[1].most());
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                    float inverse;
                    fp8::scale_of(m, sx, inverse);
                    xq[0] = v[0].quantized(inverse);
                    xq[1] = v[1].quantized(inverse);
                }
                // d0, d1: feature g, rows 2t and 2t + 1 of x; d2, d3: feature g + 8
                const float s0 = __shfl_sync(0xffffffffu, sx, 8 * t) * sw[q], s1 = __shfl_sync(0xffffffffu, sx, 8 * t + 4) * sw[q];
#pragma unroll
                for (int f = 0; f < FT; ++f) {
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 lo = u[q][f][0][h], hi = u[q][f][1][h];
                        mma_16x8x32(d, lo.x, hi.x, lo.y, hi.y, xq[h].x, xq[h].y);
                        mma_16x8x32(d, lo.z, hi.z, lo.w, hi.w, xq[h].z, xq[h].w);
                    }
                    acc[f][j][0] = fmaf(d[0], s0, acc[f][j][0]); acc[f][j][1] = fmaf(d[1], s1, acc[f][j][1]);
                    acc[f][j][2] = fmaf(d[2], s0, acc[f][j][2]); acc[f][j][3] = fmaf(d[3], s1, acc[f][j][3]);
                }
            }
        }
    }
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][16 * f + g + 8 * (i >> 1)][j * 8 + 2 * t + (i & 1)] = acc[f][j][i];
    __syncthreads();
    auto param = [&](const void* p, int64_t i, int f32) { return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); };
    for (int at = tid; at < 16 * FT * a.rows; at += 32 * kWarps) {
        const int f = at % (16 * FT), row = at / (16 * FT), col = f0 + f;
        if (col >= a.cols) continue;
        float z = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) z += sums[k][f][row];
        const int b = row / a.per_batch, r = row - b * a.per_batch;
        if (a.e.bias) z += param(a.e.bias, col, a.e.bias_f32);
        float y = a.e.act == kActGeluTanh ? activation<kActGeluTanh>(z) : a.e.act == kActGelu ? activation<kActGelu>(z)
                : a.e.act == kActSilu ? activation<kActSilu>(z) : z;
        if (a.e.gate) y *= param(a.e.gate, b * a.e.gate_stride + col, a.e.gate_f32);
        if (a.e.residual) y += param(a.e.residual, b * a.e.rs[0] + r * a.e.rs[1] + col, a.e.y_f32);
        const int64_t off = b * a.e.ys[0] + r * a.e.ys[1] + col;
        if (a.e.y_f32) static_cast<float*>(a.e.y)[off] = y;
        else static_cast<__nv_bfloat16*>(a.e.y)[off] = __float2bfloat16_rn(y);
    }
}

// ---- host side ------------------------------------------------------------------------------------
// 3-D map over [batches, rows, cols] bytes with the columns contiguous: box = 128 columns x box_rows x 1, 128-byte swizzle, what lies outside reads as zero.
inline bool make_map8(CUtensorMap* map, const Operand& o, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {cuuint64_t(o.cols), cuuint64_t(o.rows), cuuint64_t(o.batches)};
    // the stride of an axis of one entry is never used, but has to be a valid value
    const cuuint64_t row = o.rows > 1 ? cuuint64_t(o.row_stride) : cuuint64_t((o.cols + 15) / 16 * 16);
    cuuint64_t strides[2] = {row, o.batches > 1 ? cuuint64_t(o.batch_stride) : row};
    cuuint32_t box[3] = {kBlock, cuuint32_t(box_rows), 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(o.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// rows of `words` 32-bit words of exponents, one row a copy
inline bool make_map_sf(CUtensorMap* map, const void* base, int64_t rows, int words) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {cuuint64_t(words), cuuint64_t(rows), 1};
    cuuint64_t strides[2] = {cuuint64_t(words) * 4, cuuint64_t(words) * 4 * cuuint64_t(rows)};
    cuuint32_t box[3] = {cuuint32_t(words), 1, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Columns of a tile and pairs that share one: the least time by a model in nanoseconds that was fitted to launches of 40 to 3000 rows.  A pair takes 260 + 0.55
// columns per block of 128 k: an SM takes in some 92 bytes a nanosecond (with one product of each block's four left out, 333 instead of 400 ns at 224 columns), and
// below that its waits take 250 whatever the width.  Joining two pairs costs 1 to 2 us, four 2 to 4 (40 x 4096 x 1536 in 128 columns: one pair 16.9 us, two
// 13.9, four 12.5; 64 x 9216 x 1536 28.9, 20.5, 17.8).  33 clusters of 4 CTAs or 15 of 8 find room at a time.
constexpr int kLeastColumns = 64;
inline Plan plan_of8(int64_t m_tiles, int64_t cols, int64_t blocks) {
    Plan best = {kMostColumns, 1};
    double best_cost = 1e30;
    const int64_t groups = (blocks + kGroupBlocks - 1) / kGroupBlocks;
    for (int bn = kMostColumns; bn >= kLeastColumns; bn -= 32) {
        const int64_t tiles = m_tiles * ((cols + bn - 1) / bn);
        for (int splits = 1; splits <= 4; splits *= 2) {
            if ((splits == 2 && tiles > 32) || (splits == 4 && tiles > 14) || groups < splits || bn % (8 * splits)) break;
            const int64_t turns = splits > 1 ? 1 : (tiles + 73) / 74;
            const double share = splits == 1 ? double(blocks) : double((groups + splits - 1) / splits * kGroupBlocks);
            const double cost = double(turns) * std::max(share * (260 + 0.55 * bn), 500.0 + 4 * bn) + (splits == 1 ? 0 : splits == 2 ? 1800 : 3600);
            if (cost < best_cost * 0.995) { best_cost = cost; best = {bn, splits}; }
        }
    }
    return best;
}

// What a call needs besides its arguments: notes, exponents, and x in 8 bits where the call makes it.  `batches` entries of `rows`, or one of all rows; however wide the tiles are.
constexpr int kMostWCtas = 512, kMostXCtas = 148 * 8;      // that look at scales they were given (kMostXCtas, or one for each entry)
struct Room8 { int* notes; uint8_t* sfa; uint8_t* sfb; uint8_t* q; int64_t q_stride; size_t bytes; };
inline Room8 room8_of(char* p, int64_t batches, int64_t rows, int64_t cols, int64_t k, bool quantises) {
    Room8 r = {};
    size_t off = 0;
    const int64_t blocks = (k + kBlock - 1) / kBlock, groups = (blocks + kGroupBlocks - 1) / kGroupBlocks;
    const int64_t tiles = batches * ((rows + kTileM - 1) / kTileM) * 2;
    r.notes = reinterpret_cast<int*>(p + off);       off += align256(size_t(kMostWCtas + std::max<int64_t>(kMostXCtas, batches)) * 4);
    r.sfa = reinterpret_cast<uint8_t*>(p + off);     off += align256(size_t(tiles * groups) * kSfA);
    r.sfb = reinterpret_cast<uint8_t*>(p + off);     off += align256(size_t((cols + kLeastColumns - 1) / kLeastColumns * groups) * kSfB);
    if (quantises) {
        r.q_stride = blocks * kBlock;
        r.q = reinterpret_cast<uint8_t*>(p + off);   off += align256(size_t(batches * rows) * r.q_stride);
    }
    r.bytes = off;
    return r;
}

template <bool kF32, bool kRuns>
inline carnator_status launch_stages8(const Operand& A, const Operand& B, const Room8& room, Args8 a, cudaStream_t stream, char* err, size_t errlen) {
    const uint32_t stage = kABytes8 + uint32_t(a.t.bn / 2) * kBlock;
    a.t.stages = int(std::min<uint32_t>(kMaxStages, kSfAt / stage));
    static_assert(kMaxStages <= int(kSfSlots), "groups of one block: a slot of exponents is filled again when the products that read it have completed");
    CUtensorMap ma, mb, msa, msb;
    if (!make_map8(&ma, A, 128) || !make_map8(&mb, B, a.t.bn / 2) || !make_map_sf(&msa, room.sfa, int64_t(a.t.batches) * a.t.tiles_m * 2 * a.groups, int(kSfA / 4)) ||
        !make_map_sf(&msb, room.sfb, int64_t(a.t.tiles_n) * a.groups, int(kSfB / 4))) {
        snprintf(err, errlen, "cuTensorMapEncodeTiled failed or is unavailable");
        return CARNATOR_ERR_CUDA;
    }
    auto kern = linear_fp8_kernel<kF32, kRuns>;
    static SmemAllowed allowed;
    const unsigned long long ctx = context_id();
    if (!allowed.has(ctx)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemTc));
        if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(linear_fp8_kernel)", err, errlen);
        cudaFuncAttributes attr;         // the hand-over of registers only completes if the block owns them
        const cudaError_t f = cudaFuncGetAttributes(&attr, kern);
        if (f != cudaSuccess) return cuda_error(f, "cudaFuncGetAttributes(linear_fp8_kernel)", err, errlen);
        if (attr.numRegs * kThreadsTc < 128 * 40 + 256 * 208) {
            snprintf(err, errlen, "linear_fp8_kernel was built with %d registers per thread: too few for its setmaxnreg split", attr.numRegs);
            return CARNATOR_ERR_UNSUPPORTED;
        }
        allowed.add(ctx);
    }
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = unsigned(2 * a.t.splits); at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    const int clusters = a.t.splits > 1 ? a.t.tiles : std::min(a.t.tiles, 74);
    cfg.gridDim = dim3(unsigned(clusters * 2 * a.t.splits)); cfg.blockDim = dim3(kThreadsTc); cfg.dynamicSmemBytes = kSmemTc; cfg.stream = stream;
    cfg.attrs = at; cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ma, mb, msa, msb, a);
    if (e != cudaSuccess) return cuda_error(e, "linear_fp8_kernel", err, errlen);
    return CARNATOR_OK;
}

// Both kernels of a call.  `a`: everything but the plan; `p`: x, scales and header; A: x in 8 bits.
inline carnator_status launch_product8(const Operand& A, const Operand& B, const Room8& room, Args8 a, PrepareArgs p, int type, cudaStream_t stream, char* err, size_t errlen) {
    a.t.k_batches = 1;
    a.t.k_tiles = ceil_div(a.t.k_len, kBlock);
    a.groups = ceil_div(a.t.k_tiles, kGroupBlocks);
    a.t.tiles_m = ceil_div(a.t.rows, kTileM);
    const Plan plan = plan_of8(int64_t(a.t.batches) * a.t.tiles_m, a.t.cols, a.t.k_tiles);
    a.t.bn = plan.bn; a.t.splits = plan.splits;
    a.t.tiles_n = ceil_div(a.t.cols, a.t.bn);
    const int64_t tiles = int64_t(a.t.batches) * a.t.tiles_m * a.t.tiles_n;
    if (tiles > (int64_t(1) << 30) || int64_t(a.t.batches) * a.t.tiles_m * 2 * a.groups > (int64_t(1) << 30) || int64_t(a.t.tiles_n) * a.groups > (int64_t(1) << 30))
        return CARNATOR_ERR_UNSUPPORTED;
    a.t.tiles = int(tiles);
    a.t.group_m = 8;

    p.q.batches = a.t.batches; p.q.rows = a.t.rows; p.q.cols = a.t.k_len; p.q.blocks = a.t.k_tiles;
    p.sfa = room.sfa; p.sfb = room.sfb; p.notes = room.notes; p.hdr = a.t.hdr;
    p.groups = a.groups; p.row_tiles = a.t.tiles_m * 2;
    p.cols = a.t.cols; p.bn = a.t.bn; p.tiles_n = a.t.tiles_n;
    p.x_ctas = type == kXE4m3 ? int(std::min<int64_t>(std::max(kMostXCtas / a.t.batches, 1), (int64_t(a.groups) * a.t.rows + fp8::kRowThreads - 1) / fp8::kRowThreads))
                              : std::min(fp8::row_ctas(p.q, type == kXF32), std::max((1 << 30) / a.t.batches, 1));
    p.w_ctas = int(std::min<int64_t>(kMostWCtas, int64_t(a.t.tiles_n) * a.groups));
    const dim3 grid(unsigned(p.x_ctas * a.t.batches + p.w_ctas));
    const cudaError_t e = type == kXBf16 ? launch_dependent(prepare_fp8_kernel<kXBf16>, grid, dim3(fp8::kRowThreads), 0, stream, p)
                        : type == kXF32  ? launch_dependent(prepare_fp8_kernel<kXF32>, grid, dim3(fp8::kRowThreads), 0, stream, p)
                                         : launch_dependent(prepare_fp8_kernel<kXE4m3>, grid, dim3(fp8::kRowThreads), 0, stream, p);
    if (e != cudaSuccess) return cuda_error(e, "prepare_fp8_kernel", err, errlen);
    a.notes = room.notes; a.n_notes = p.w_ctas + (type == kXE4m3 ? p.x_ctas * a.t.batches : 0);
    a.sfa = room.sfa;
    // whether a pair's share of k is longer than one accumulator may sum up
    const int64_t share = int64_t((a.groups + a.t.splits - 1) / a.t.splits) * kGroupBlocks * kBlock;
    if (a.t.e.y_f32)
        return share > kLongRun ? launch_stages8<true, true>(A, B, room, a, stream, err, errlen) : launch_stages8<true, false>(A, B, room, a, stream, err, errlen);
    return share > kLongRunBf16 ? launch_stages8<false, true>(A, B, room, a, stream, err, errlen) : launch_stages8<false, false>(A, B, room, a, stream, err, errlen);
}

template <int NT, int kType>
inline cudaError_t launch_rows8_warps(const RowsArgs8& a, cudaStream_t stream) {
    const int grid = ceil_div(a.cols, 16);
    auto run = [&](void (*kernel)(RowsArgs8), int ft, int warps) { return launch_dependent(kernel, dim3(unsigned(ceil_div(a.cols, 16 * ft))), dim3(unsigned(32 * warps)), 0, stream, a); };
    // Many warps share k where there are few CTAs, so that all of W is on its way at once; where CTAs fill the SMs several times over, tiles share x, which every CTA
    // takes to 8 bits for itself.  us (1 row, cold W; tiles x warps): 1536 x 1536 1x16 3.0, 2x16 3.8; 1536 x 8960 2x8 5.6, 1x8 7.9; 5120 x 5120 2x8 12.3, 1x8 12.4,
    // 4x8 17.9; 5120 x 13824 4x8 20.8, 2x8 24.0, 4x4 31.5; 5120 x 30720 4x4 37.9, 4x8 40.7, 1x4 43.9.
    if (grid <= 148) return run(linear_fp8_rows_kernel<NT, 16, kType, 1>, 1, 16);
    if (grid <= 4 * 148) return run(linear_fp8_rows_kernel<NT, 8, kType, 2>, 2, 8);
    if (grid <= 8 * 148) return run(linear_fp8_rows_kernel<NT, 8, kType, 4>, 4, 8);
    return run(linear_fp8_rows_kernel<NT, 4, kType, 4>, 4, 4);
}
template <int kType>
inline cudaError_t launch_rows8(const RowsArgs8& a, cudaStream_t stream) {
    return a.rows <= 8 ? launch_rows8_warps<1, kType>(a, stream) : launch_rows8_warps<2, kType>(a, stream);
}

}  // namespace lin8
}  // namespace carnator
