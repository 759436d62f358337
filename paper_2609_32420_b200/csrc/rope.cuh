// Rotary positions: the channels of a head in pairs (u, v), pair i turned by the angle of its token's position on the pair's axis,
//   th = pos[axis(i)] f_i,   (u, v) -> m (u cos th - v sin th, u sin th + v cos th);
// the transposed turn (-th) is its gradient.  The channels of pair i are 2i and 2i + 1, or i and i + pairs.
//
// Bound by memory: every value is read and written once.  A thread has one unit of a token's channels and walks over the heads, several of them on their way
// at a time, so that the angles, which all heads share, are computed once per token and stay in registers.  Angles are taken in 64 bits, in turns: the
// position times f_i / 2 pi, less the nearest whole number, is at most 1/2 and loses nothing to the size of the position (at position 10^6 a 32-bit product is off
// by up to 0.06 radians); sine and cosine of its first 32 bits are CUDA's.
// 75600 x 80 heads of 128 in bf16: 471 us, the copy rate.
#pragma once
#include "norm.cuh"

namespace carnator {
namespace rope {

constexpr int kThreads = 256;
constexpr int kMaxHead = 256;            // a token's units fit a CTA

struct Args {
    const void* x; void* y;
    const double* freq;                  // [pairs] radians per position
    const int32_t* pos;                  // [B,N,axes] or NULL: text tokens (which do not turn), then the grid
    int64_t xs[3], ys[3];                // (batch, head, token)
    int64_t ps[2];                       // (batch, token)
    int H, N, D, axes;
    int n_text, Hg, Wg;
    int offset[3];
    int pairs, end0, end1;               // all pairs; where the pairs of the second and of the third axis begin
    int units, tile, splits;             // units of a token, tokens of a CTA, CTAs that share the heads of their tokens
    int in_place;                        // what does not turn stays as it is
    float amplitude, sign;
};

// VEC elements of a row, of which n are there
template <bool F32, int VEC>
struct Piece {
    static constexpr int kBytes = VEC * (F32 ? 4 : 2), kWords = kBytes > 4 ? kBytes / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* base, int64_t off, int n) {
        const char* p = static_cast<const char*>(base) + off * (F32 ? 4 : 2);
        if (n >= VEC) {
            if constexpr (kBytes >= 16) {
#pragma unroll
                for (int i = 0; i < kBytes / 16; ++i)
                    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "l"(p + 16 * i));
            } else if constexpr (kBytes == 8) {
                asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
            } else if constexpr (kBytes == 4) {
                asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
            } else {
                w[0] = *reinterpret_cast<const volatile uint16_t*>(p);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < n) {
                    if (F32) w[F32 ? i : 0] = reinterpret_cast<const volatile uint32_t*>(p)[i];
                    else w[i / 2] |= uint32_t(reinterpret_cast<const volatile uint16_t*>(p)[i]) << (16 * (i & 1));
                }
        }
    }
    __device__ __forceinline__ void store(void* base, int64_t off, int n) const {
        char* p = static_cast<char*>(base) + off * (F32 ? 4 : 2);
        if (n >= VEC) {
            if constexpr (kBytes >= 16) {
#pragma unroll
                for (int i = 0; i < kBytes / 16; ++i)
                    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p + 16 * i), "r"(w[4 * i]), "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3]));
            } else if constexpr (kBytes == 8) {
                asm volatile("st.global.v2.b32 [%0], {%1, %2};" ::"l"(p), "r"(w[0]), "r"(w[1]));
            } else if constexpr (kBytes == 4) {
                asm volatile("st.global.b32 [%0], %1;" ::"l"(p), "r"(w[0]));
            } else {
                *reinterpret_cast<volatile uint16_t*>(p) = uint16_t(w[0]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < n) {
                    if (F32) reinterpret_cast<volatile uint32_t*>(p)[i] = w[F32 ? i : 0];
                    else reinterpret_cast<volatile uint16_t*>(p)[i] = uint16_t(w[i / 2] >> (16 * (i & 1)));
                }
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if (F32) return __uint_as_float(w[F32 ? i : 0]);
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    // two neighbours
    __device__ __forceinline__ void set2(int i, float lo, float hi) {
        if (F32) { w[F32 ? i : 0] = __float_as_uint(lo); w[F32 && VEC > 1 ? i + 1 : 0] = __float_as_uint(hi); }
        else w[i / 2] = norm::pack_bf16(lo, hi);
    }
    __device__ __forceinline__ void set1(float v) { w[0] = F32 ? __float_as_uint(v) : norm::pack_bf16(v, 0.f); }
};

// cosine and sine of pair i of a token, times the amplitude
struct Token {
    double at[3];
    __device__ __forceinline__ Token(const Args& a, int b, int n) {
        if (a.pos) {
            const int32_t* p = a.pos + b * a.ps[0] + n * a.ps[1];
#pragma unroll
            for (int k = 0; k < 3; ++k) at[k] = k < a.axes ? double(p[k]) + double(a.offset[k]) : 0.0;
        } else {
            const int g = n - a.n_text, row = g / a.Wg, f = row / a.Hg;
            at[0] = double(f) + double(a.offset[0]);
            at[1] = double(row - f * a.Hg) + double(a.offset[1]);
            at[2] = double(g - row * a.Wg) + double(a.offset[2]);
        }
    }
    __device__ __forceinline__ void turn(const Args& a, int i, float& c, float& s) const {
        // position x frequency / 2 pi with what either product's rounding leaves (1 / 2 pi in two parts), less the nearest whole number: nothing is lost to the size of the position
        constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;
        const double p = i < a.end0 ? at[0] : i < a.end1 ? at[1] : at[2], f = a.freq[i];
        const double th = __dmul_rn(p, f), turns = __dmul_rn(th, kTurn);
        const double part = turns - rint(turns) + fma(th, kTurn, -turns) + fma(th, kTurnRest, fma(p, f, -th) * kTurn);
        // sine and cosine of 32 bits of it, and the rest by their slopes
        const float hi = float(part), lo = float(part - hi) * 6.2831853f;
        float sn, cs;
        sincospif(2.f * hi, &sn, &cs);
        c = a.amplitude * fmaf(-lo, sn, cs);
        s = a.amplitude * a.sign * fmaf(lo, cs, sn);
    }
};

__device__ __forceinline__ bool place(const Args& a, int& unit, int& n, int& h0, int& h1) {
    const int t = threadIdx.x / a.units, part = int(blockIdx.x) % a.splits;
    unit = threadIdx.x - t * a.units;
    n = int(blockIdx.x) / a.splits * a.tile + t;
    h0 = int(int64_t(a.H) * part / a.splits);
    h1 = int(int64_t(a.H) * (part + 1) / a.splits);
    return t < a.tile && n < a.N;
}

// Neighbours: a unit is 8 channels, 4 pairs.
template <bool F32, int HEADS>
__global__ void __launch_bounds__(kThreads) rope_neighbours_kernel(const Args a) {
    int unit, n, h0, h1;
    grid_launch_dependents();
    grid_wait();
    if (!place(a, unit, n, h0, h1)) return;
    const int b = blockIdx.y, ch = unit * 8, left = min(a.D - ch, 8), on = (a.pos || n >= a.n_text) ? min(a.pairs - unit * 4, 4) : 0;
    if (a.in_place && on <= 0) return;
    int64_t xo = b * a.xs[0] + n * a.xs[2] + ch + h0 * a.xs[1], yo = b * a.ys[0] + n * a.ys[2] + ch + h0 * a.ys[1];
    Piece<F32, 8> p[HEADS];
    int h = h0;
    auto fetch = [&]() {                 // ahead of the angles
#pragma unroll
        for (int k = 0; k < HEADS; ++k) if (h + k < h1) p[k].load(a.x, xo + k * a.xs[1], left);
    };
    fetch();
    float c[4], s[4];
    if (on > 0) {
        const Token t(a, b, n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < on) t.turn(a, unit * 4 + i, c[i], s[i]);
    }
    while (true) {
#pragma unroll
        for (int k = 0; k < HEADS; ++k)
            if (h + k < h1) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < on) {
                        const float u = p[k].get(2 * i), v = p[k].get(2 * i + 1);
                        p[k].set2(2 * i, u * c[i] - v * s[i], u * s[i] + v * c[i]);
                    }
                p[k].store(a.y, yo + k * a.ys[1], left);
            }
        h += HEADS;
        if (h >= h1) break;
        xo += HEADS * a.xs[1];
        yo += HEADS * a.ys[1];
        fetch();
    }
}

// Halves: a unit is VEC pairs, VEC channels of either half; behind them VEC channels that do not turn.  VEC: the most that divides the number of
// pairs, so that both halves start on its boundary.
template <bool F32, int VEC, int HEADS>
__global__ void __launch_bounds__(kThreads) rope_halves_kernel(const Args a) {
    int unit, n, h0, h1;
    grid_launch_dependents();
    grid_wait();
    if (!place(a, unit, n, h0, h1)) return;
    const int b = blockIdx.y, turning = a.pairs / VEC;
    const bool pair = unit < turning, on = pair && (a.pos || n >= a.n_text);
    if (a.in_place && !on) return;
    const int ch = pair ? unit * VEC : 2 * a.pairs + (unit - turning) * VEC, left = pair ? VEC : a.D - ch;
    int64_t xo = b * a.xs[0] + n * a.xs[2] + ch + h0 * a.xs[1], yo = b * a.ys[0] + n * a.ys[2] + ch + h0 * a.ys[1];
    Piece<F32, VEC> p[HEADS], q[HEADS];
    int h = h0;
    auto fetch = [&]() {
#pragma unroll
        for (int k = 0; k < HEADS; ++k)
            if (h + k < h1) {
                p[k].load(a.x, xo + k * a.xs[1], left);
                if (pair) q[k].load(a.x, xo + k * a.xs[1] + a.pairs, VEC);
            }
    };
    fetch();
    float c[VEC], s[VEC];
    if (on) {
        const Token t(a, b, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) t.turn(a, unit * VEC + i, c[i], s[i]);
    }
    while (true) {
#pragma unroll
        for (int k = 0; k < HEADS; ++k)
            if (h + k < h1) {
                if (on) {
                    if constexpr (VEC == 1) {
                        const float u = p[k].get(0), v = q[k].get(0);
                        p[k].set1(u * c[0] - v * s[0]);
                        q[k].set1(u * s[0] + v * c[0]);
                    } else {
#pragma unroll
                        for (int i = 0; i < VEC; i += 2) {
                            const float u0 = p[k].get(i), u1 = p[k].get(i + 1), v0 = q[k].get(i), v1 = q[k].get(i + 1);
                            p[k].set2(i, u0 * c[i] - v0 * s[i], u1 * c[i + 1] - v1 * s[i + 1]);
                            q[k].set2(i, u0 * s[i] + v0 * c[i], u1 * s[i + 1] + v1 * c[i + 1]);
                        }
                    }
                }
                p[k].store(a.y, yo + k * a.ys[1], left);
                if (pair) q[k].store(a.y, yo + k * a.ys[1] + a.pairs, VEC);
            }
        h += HEADS;
        if (h >= h1) break;
        xo += HEADS * a.xs[1];
        yo += HEADS * a.ys[1];
        fetch();
    }
}

// Halves whose channels come in whole pieces of 8, of a head of 8, 16, .. 256 channels: a lane has 8 neighbouring channels, as they lie in memory, and takes the other half of its
// pairs from the lane that has it.  (2 x 17776 x 24 heads of 64, of which 48 channels turn: 38.9 us; 43.7 with pieces of both halves in one lane, which
// touch parts of sectors.)
template <bool F32, int HEADS>
__global__ void __launch_bounds__(kThreads) rope_halves_across_kernel(const Args a) {
    int unit, n, h0, h1;
    grid_launch_dependents();
    grid_wait();
    const bool there = place(a, unit, n, h0, h1);
    const int b = blockIdx.y, half = a.pairs / 8;        // units of a half
    const bool turns = unit < 2 * half, on = there && turns && (a.pos || n >= a.n_text), moves = there && (on || !a.in_place);
    const int first = turns && unit >= half ? unit - half : unit, other = int(threadIdx.x & 31) + (!turns ? 0 : unit >= half ? -half : half);
    int64_t xo = b * a.xs[0] + n * a.xs[2] + unit * 8 + h0 * a.xs[1], yo = b * a.ys[0] + n * a.ys[2] + unit * 8 + h0 * a.ys[1];
    Piece<F32, 8> p[HEADS];
    int h = h0;
    auto fetch = [&]() {
#pragma unroll
        for (int k = 0; k < HEADS; ++k) if (moves && h + k < h1) p[k].load(a.x, xo + k * a.xs[1], 8);
    };
    fetch();
    float c[8], s[8];
    if (on) {
        const Token t(a, b, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.turn(a, first * 8 + i, c[i], s[i]);
            if (unit < half) s[i] = -s[i];           // u cos - v sin here, v cos + u sin in the other half
        }
    }
    while (true) {                       // the same trips for every lane
#pragma unroll
        for (int k = 0; k < HEADS; ++k)
            if (h + k < h1) {
                Piece<F32, 8> q;
#pragma unroll
                for (int i = 0; i < Piece<F32, 8>::kWords; ++i) q.w[i] = __shfl_sync(0xffffffffu, p[k].w[i], other);
                if (on) {
#pragma unroll
                    for (int i = 0; i < 8; i += 2) p[k].set2(i, p[k].get(i) * c[i] + q.get(i) * s[i], p[k].get(i + 1) * c[i + 1] + q.get(i + 1) * s[i + 1]);
                }
                if (moves) p[k].store(a.y, yo + k * a.ys[1], 8);
            }
        h += HEADS;
        if (h >= h1) break;
        xo += HEADS * a.xs[1];
        yo += HEADS * a.ys[1];
        fetch();
    }
}

// ---- host side ------------------------------------------------------------------------------------
template <bool F32>
inline cudaError_t launch(Args a, int B, bool half, cudaStream_t stream) {
    const int vec = !half ? 8 : a.pairs % 8 == 0 ? 8 : a.pairs % 4 == 0 ? 4 : a.pairs % 2 == 0 ? 2 : 1;
    const bool across = half && vec == 8 && a.D >= 8 && (a.D & (a.D - 1)) == 0;      // a token's lanes lie within a warp
    a.units = half && !across ? a.pairs / vec + ceil_div(a.D - 2 * a.pairs, vec) : ceil_div(a.D, 8);
    a.tile = kThreads / a.units;
    if (a.tile > a.N) a.tile = a.N;
    // enough CTAs for every SM; the angles are computed again by each that shares a token
    const int64_t tiles = int64_t(ceil_div(a.N, a.tile));
    a.splits = int(std::min<int64_t>(a.H, std::max<int64_t>(1, 148 * 8 / (tiles * B))));
    const dim3 grid(unsigned(tiles * a.splits), unsigned(B)), block(unsigned((a.tile * a.units + 31) / 32 * 32));
    auto run = [&](void (*kernel)(Args)) { return launch_dependent(kernel, grid, block, 0, stream, a); };
    if (!half) return run(rope_neighbours_kernel<F32, F32 ? 4 : 8>);
    if (across) return run(rope_halves_across_kernel<F32, F32 ? 4 : 8>);
    if (vec == 8) return run(rope_halves_kernel<F32, 8, F32 ? 2 : 4>);
    if (vec == 4) return run(rope_halves_kernel<F32, 4, 4>);
    return vec == 2 ? run(rope_halves_kernel<F32, 2, 8>) : run(rope_halves_kernel<F32, 1, 8>);
}

}  // namespace rope
}  // namespace carnator
