// C-ABI entry points between a layer's attention, its projections and the residual stream: rotary positions, block norms, 8-bit operands and their product.
#define CARNATOR_NO_ATTENTION_KERNELS
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "carnator.h"
#include "api.h"
#include "rope.cuh"
#include "block_norm.cuh"
#include "fp8_quantize.cuh"
#include "linear_fp8.cuh"

using namespace carnator;

namespace {
constexpr int64_t kMostStride = int64_t(1) << 38;

void count_launch() { g_launches.fetch_add(1, std::memory_order_relaxed); }

// ------------------------------------------------------------------------------------------------
// rotary positions
// ------------------------------------------------------------------------------------------------
carnator_status check_rope_shape(const carnator_rope_shape* s, bool positions) {
    if (!s || s->B <= 0 || s->H <= 0 || s->N <= 0 || s->D <= 0) return CARNATOR_ERR_INVALID_ARG;
    if (!dtype_ok(s->x_dtype) || (s->layout != CARNATOR_ROPE_INTERLEAVED && s->layout != CARNATOR_ROPE_HALF)) return CARNATOR_ERR_INVALID_ARG;
    if (!std::isfinite(s->amplitude)) return CARNATOR_ERR_INVALID_ARG;
    int64_t pairs = 0;
    for (int p : s->pairs) {
        if (p < 0) return CARNATOR_ERR_INVALID_ARG;
        pairs += p;
    }
    if (pairs == 0 || 2 * pairs > s->D) return CARNATOR_ERR_INVALID_ARG;
    if (positions) {
        if (s->axes < 1 || s->axes > 3) return CARNATOR_ERR_INVALID_ARG;
        for (int i = s->axes; i < 3; ++i) if (s->pairs[i]) return CARNATOR_ERR_INVALID_ARG;
        if ((s->B > 1 && (s->pos_stride[0] < 0 || s->pos_stride[0] > kMostStride)) || (s->N > 1 && (s->pos_stride[1] < 0 || s->pos_stride[1] > kMostStride))) return CARNATOR_ERR_INVALID_ARG;
    } else {
        if (s->axes != 0) return CARNATOR_ERR_INVALID_ARG;       // a record of positions whose call has forgotten them
        if (s->n_text < 0 || s->T < 0 || s->Hg < 0 || s->Wg < 0) return CARNATOR_ERR_INVALID_ARG;
        const int64_t frame = int64_t(s->Hg) * s->Wg;            // below 2^62
        const int64_t video = int64_t(s->N) - s->n_text;
        if (s->T == 0 || frame == 0 ? video != 0 : (frame > video || video % frame || video / frame != s->T)) return CARNATOR_ERR_INVALID_ARG;
    }
    if (s->D > rope::kMaxHead || s->B > 65535 || s->H > 65535 || s->N > (1 << 27)) return CARNATOR_ERR_UNSUPPORTED;
    return CARNATOR_OK;
}
}  // namespace

extern "C" carnator_status carnator_rope_frequencies(const carnator_rope_scaling* s, double* freq, double* amplitude_opt) {
    if (!s || !freq || !(s->theta > 1) || !std::isfinite(s->theta) || s->mode < CARNATOR_ROPE_SCALE_NONE || s->mode > CARNATOR_ROPE_SCALE_RAMP) return CARNATOR_ERR_INVALID_ARG;
    const bool ramp = s->mode == CARNATOR_ROPE_SCALE_RAMP;
    if (ramp && !(s->low >= 0 && s->high > s->low && std::isfinite(s->high))) return CARNATOR_ERR_INVALID_ARG;
    double most = 1;
    for (int a = 0; a < 3; ++a) {
        if (s->pairs[a] < 0 || s->pairs[a] > (1 << 20)) return CARNATOR_ERR_INVALID_ARG;
        if (s->pairs[a] == 0 || s->mode == CARNATOR_ROPE_SCALE_NONE) continue;
        if (!(s->factor[a] >= 1) || !std::isfinite(s->factor[a]) || (ramp && !(s->original[a] > 0 && std::isfinite(s->original[a])))) return CARNATOR_ERR_INVALID_ARG;
        most = std::max(most, s->factor[a]);
    }
    int at = 0;
    for (int a = 0; a < 3; ++a) {
        const double n = s->pairs[a];
        double theta = s->theta;
        if (s->mode == CARNATOR_ROPE_SCALE_BASE && s->pairs[a] > 1) theta *= std::pow(s->factor[a], n / (n - 1));
        for (int i = 0; i < s->pairs[a]; ++i) {
            double f = std::pow(theta, -i / n);
            if (s->mode == CARNATOR_ROPE_SCALE_LINEAR) f /= s->factor[a];
            if (ramp) {
                const double turns = s->original[a] * f / (2 * M_PI), g = std::min(std::max((turns - s->low) / (s->high - s->low), 0.0), 1.0);
                f *= g + (1 - g) / s->factor[a];
            }
            freq[at++] = f;
        }
    }
    if (amplitude_opt) *amplitude_opt = ramp ? 0.1 * std::log(most) + 1 : 1;
    return CARNATOR_OK;
}

extern "C" carnator_status carnator_rope(const void* X, const double* freq, const int32_t* positions, const carnator_rope_shape* s, void* Y, void* stream_) {
    carnator_status st = check_rope_shape(s, positions != nullptr);
    if (st != CARNATOR_OK) return st;
    if (!X || !Y || !freq || !aligned(X, 16) || !aligned(Y, 16) || !aligned(freq, 8) || !aligned(positions, 4)) return CARNATOR_ERR_INVALID_ARG;
    const int64_t size[3] = {s->B, s->H, s->N};
    if (!axes_ok(s->x_stride, size, 3, s->D, s->x_dtype, false, false) || !axes_ok(s->y_stride, size, 3, s->D, s->x_dtype, true, false)) return CARNATOR_ERR_INVALID_ARG;
    st = check_device();
    if (st != CARNATOR_OK) return st;
    rope::Args a = {};
    a.x = X; a.y = Y; a.freq = freq; a.pos = positions;
    a.in_place = X == Y;
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = size[i] == 1 ? 0 : s->x_stride[i];
        a.ys[i] = size[i] == 1 ? 0 : s->y_stride[i];
        if (a.xs[i] != a.ys[i]) a.in_place = 0;
        a.offset[i] = s->offset[i];
    }
    a.ps[0] = s->B == 1 ? 0 : s->pos_stride[0]; a.ps[1] = s->N == 1 ? 0 : s->pos_stride[1];
    a.H = s->H; a.N = s->N; a.D = s->D; a.axes = s->axes;
    a.n_text = s->n_text; a.Hg = std::max(s->Hg, 1); a.Wg = std::max(s->Wg, 1);
    a.end0 = s->pairs[0]; a.end1 = s->pairs[0] + s->pairs[1]; a.pairs = a.end1 + s->pairs[2];
    a.amplitude = s->amplitude; a.sign = s->inverse ? -1.f : 1.f;
    const bool half = s->layout == CARNATOR_ROPE_HALF;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const cudaError_t e = s->x_dtype == CARNATOR_DTYPE_F32 ? rope::launch<true>(a, s->B, half, stream) : rope::launch<false>(a, s->B, half, stream);
    if (e != cudaSuccess) return cuda_fail(e, "rope kernel");
    count_launch();
    return CARNATOR_OK;
}

// ------------------------------------------------------------------------------------------------
// block norms
// ------------------------------------------------------------------------------------------------
namespace {
carnator_status check_block_shape(const carnator_block_norm_shape* s) {
    if (!s || s->B <= 0 || s->N <= 0 || s->C <= 0) return CARNATOR_ERR_INVALID_ARG;
    if (s->post < CARNATOR_NORM_NONE || s->post > CARNATOR_NORM_RMS || s->pre < CARNATOR_NORM_LAYER || s->pre > CARNATOR_NORM_RMS) return CARNATOR_ERR_INVALID_ARG;
    if (!dtype_ok(s->stream_dtype) || !dtype_ok(s->x_dtype) || !dtype_ok(s->y_dtype) || !dtype_ok(s->weight_dtype) || !dtype_ok(s->mod_dtype)) return CARNATOR_ERR_INVALID_ARG;
    if (!(s->post_eps >= 0.f) || std::isinf(s->post_eps) || !(s->eps >= 0.f) || std::isinf(s->eps) || !std::isfinite(s->residual_scale)) return CARNATOR_ERR_INVALID_ARG;
    if (s->gate_stride < 0 || s->shift_stride < 0 || s->scale_stride < 0) return CARNATOR_ERR_INVALID_ARG;
    if (s->C > blk::kMostChannels || s->B > 65535 || int64_t(s->B) * s->N > (int64_t(1) << 30)) return CARNATOR_ERR_UNSUPPORTED;
    return CARNATOR_OK;
}
bool block_axes_ok(const carnator_block_norm_shape* s, const int64_t st[2], int32_t dtype, bool written) {
    const int64_t size[2] = {s->B, s->N};
    return axes_ok(st, size, 2, s->C, dtype, written, false);
}
bool block_vectors_ok(const carnator_block_norm_shape* s, const void* w1, const void* b1, const void* w2, const void* b2, const void* gate, const void* shift, const void* scale) {
    const size_t w = size_t(dtype_bytes(s->weight_dtype)), m = size_t(dtype_bytes(s->mod_dtype));
    return aligned(w1, w) && aligned(b1, w) && aligned(w2, w) && aligned(b2, w) && aligned(gate, m) && aligned(shift, m) && aligned(scale, m);
}
// Strides as the kernels take them (that of an axis of one entry may be anything), parameters, what may be read 16 bytes at a time.
void block_args(const carnator_block_norm_shape* s, blk::Args2& a, const void* w1, const void* b1, const void* gate, const void* w2, const void* b2, const void* shift, const void* scale) {
    a.w1 = w1; a.b1 = b1; a.gate = gate; a.w2 = w2; a.b2 = b2; a.shift = shift; a.scale = scale;
    a.gate_stride = s->B == 1 ? 0 : s->gate_stride; a.shift_stride = s->B == 1 ? 0 : s->shift_stride; a.scale_stride = s->B == 1 ? 0 : s->scale_stride;
    a.B = s->B; a.N = s->N; a.C = s->C;
    a.post = s->post; a.pre = s->pre;
    a.w_f32 = s->weight_dtype == CARNATOR_DTYPE_F32; a.mod_f32 = s->mod_dtype == CARNATOR_DTYPE_F32;
    a.vec_ok = vec16(w1, 0, s->weight_dtype) && vec16(b1, 0, s->weight_dtype) && vec16(w2, 0, s->weight_dtype) && vec16(b2, 0, s->weight_dtype) &&
               vec16(gate, a.gate_stride, s->mod_dtype) && vec16(shift, a.shift_stride, s->mod_dtype) && vec16(scale, a.scale_stride, s->mod_dtype);
    a.alpha = s->residual_scale; a.eps1 = s->post_eps; a.eps2 = s->eps; a.inv_c = 1.0f / float(s->C);
}
void block_strides(const carnator_block_norm_shape* s, int64_t (&to)[2], const int64_t (&from)[2]) {
    to[0] = s->B == 1 ? 0 : from[0];
    to[1] = s->N == 1 ? 0 : from[1];
}
}  // namespace

extern "C" carnator_status carnator_block_norm(const void* R, const void* X, const void* post_weight, const void* post_bias, const void* gate,
                                               const void* weight, const void* bias, const void* shift, const void* scale,
                                               const carnator_block_norm_shape* s, void* S, void* Y, float* stats_opt, void* stream_) {
    carnator_status st = check_block_shape(s);
    if (st != CARNATOR_OK) return st;
    if (!R || !X || !S || !Y || !aligned(R, 16) || !aligned(X, 16) || !aligned(S, 16) || !aligned(Y, 16) || !aligned(stats_opt, 4)) return CARNATOR_ERR_INVALID_ARG;
    if (!block_vectors_ok(s, post_weight, post_bias, weight, bias, gate, shift, scale)) return CARNATOR_ERR_INVALID_ARG;
    if (!block_axes_ok(s, s->r_stride, s->stream_dtype, false) || !block_axes_ok(s, s->x_stride, s->x_dtype, false) || !block_axes_ok(s, s->s_stride, s->stream_dtype, true) ||
        !block_axes_ok(s, s->y_stride, s->y_dtype, true)) return CARNATOR_ERR_INVALID_ARG;
    st = check_device();
    if (st != CARNATOR_OK) return st;
    blk::Args2 a = {};
    block_args(s, a, post_weight, post_bias, gate, weight, bias, shift, scale);
    a.r = R; a.x = X; a.s = S; a.y = Y; a.stats = stats_opt;
    block_strides(s, a.rs, s->r_stride); block_strides(s, a.xs, s->x_stride); block_strides(s, a.ss, s->s_stride); block_strides(s, a.ys, s->y_stride);
    a.wide_s = rows32(S, a.ss, s->stream_dtype); a.wide_y = rows32(Y, a.ys, s->y_dtype);
    const blk::Form2 f = blk::form2_of(s->C, false);
    a.chunks = blk::chunks2_of(f, s->B, s->C, s->N, false);
    const cudaError_t e = blk::launch2<false>(a, f, s->stream_dtype == CARNATOR_DTYPE_F32, s->x_dtype == CARNATOR_DTYPE_F32, s->y_dtype == CARNATOR_DTYPE_F32,
                                              static_cast<cudaStream_t>(stream_));
    if (e != cudaSuccess) return cuda_fail(e, "block_forward_kernel");
    count_launch();
    return CARNATOR_OK;
}

extern "C" size_t carnator_block_norm_backward_workspace_bytes(const carnator_block_norm_shape* s) {
    if (check_block_shape(s) != CARNATOR_OK) return 0;
    return align256(size_t(s->B) * blk::chunks2_of(blk::form2_of(s->C, true), s->B, s->C, s->N, true) * 4 * s->C * 4);
}

extern "C" carnator_status carnator_block_norm_backward(const void* dY, const void* dS_opt, const void* S, const void* X, const float* stats,
                                                        const void* post_weight, const void* post_bias, const void* gate,
                                                        const void* weight, const void* bias, const void* scale,
                                                        const carnator_block_norm_shape* s, void* dR, void* dX,
                                                        float* dpost_weight_opt, float* dpost_bias_opt, float* dgate_opt,
                                                        float* dweight_opt, float* dbias_opt, float* dshift_opt, float* dscale_opt,
                                                        void* ws, size_t ws_bytes, void* stream_) {
    carnator_status st = check_block_shape(s);
    if (st != CARNATOR_OK) return st;
    if (!dY || !S || !X || !stats || !dR || !dX) return CARNATOR_ERR_INVALID_ARG;
    if (!aligned(dY, 16) || !aligned(dS_opt, 16) || !aligned(S, 16) || !aligned(X, 16) || !aligned(dR, 16) || !aligned(dX, 16) || !aligned(stats, 4)) return CARNATOR_ERR_INVALID_ARG;
    float* const wanted[7] = {dpost_weight_opt, dpost_bias_opt, dgate_opt, dweight_opt, dbias_opt, dshift_opt, dscale_opt};
    bool sums = false;
    for (float* p : wanted) {
        if (!aligned(p, 4)) return CARNATOR_ERR_INVALID_ARG;
        sums = sums || p;
    }
    if (!block_vectors_ok(s, post_weight, post_bias, weight, bias, gate, nullptr, scale)) return CARNATOR_ERR_INVALID_ARG;
    if (!block_axes_ok(s, s->y_stride, s->y_dtype, false) || (dS_opt && !block_axes_ok(s, s->ds_stride, s->stream_dtype, false)) ||
        !block_axes_ok(s, s->s_stride, s->stream_dtype, false) || !block_axes_ok(s, s->x_stride, s->x_dtype, false) ||
        !block_axes_ok(s, s->dr_stride, s->stream_dtype, true) || !block_axes_ok(s, s->dx_stride, s->x_dtype, true)) return CARNATOR_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < carnator_block_norm_backward_workspace_bytes(s)) return CARNATOR_ERR_WORKSPACE;
    st = check_device();
    if (st != CARNATOR_OK) return st;
    blk::Args2 a = {};
    block_args(s, a, post_weight, nullptr, gate, weight, nullptr, nullptr, scale);
    a.dy = dY; a.r = dS_opt; a.s = const_cast<void*>(S); a.x = X; a.dr = dR; a.dx = dX;
    a.stats = const_cast<float*>(stats);
    a.part = sums ? static_cast<float*>(ws) : nullptr;
    block_strides(s, a.dys, s->y_stride); block_strides(s, a.rs, s->ds_stride); block_strides(s, a.ss, s->s_stride); block_strides(s, a.xs, s->x_stride);
    block_strides(s, a.drs, s->dr_stride); block_strides(s, a.dxs, s->dx_stride);
    a.wide_s = rows32(dR, a.drs, s->stream_dtype); a.wide_dx = rows32(dX, a.dxs, s->x_dtype);
    const blk::Form2 f = blk::form2_of(s->C, true);
    a.chunks = blk::chunks2_of(f, s->B, s->C, s->N, true);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const cudaError_t e = blk::launch2<true>(a, f, s->stream_dtype == CARNATOR_DTYPE_F32, s->x_dtype == CARNATOR_DTYPE_F32, s->y_dtype == CARNATOR_DTYPE_F32, stream);
    if (e != cudaSuccess) return cuda_fail(e, "block_backward_kernel");
    count_launch();
    if (!sums) return CARNATOR_OK;
    blk::ReduceArgs2 r = {};
    r.part = a.part;
    r.w1 = post_weight; r.b1 = post_bias; r.gate = gate; r.w2 = weight; r.b2 = bias; r.scale = scale;
    r.dw1 = dpost_weight_opt; r.db1 = dpost_bias_opt; r.dgate = dgate_opt; r.dw2 = dweight_opt; r.db2 = dbias_opt; r.dshift = dshift_opt; r.dscale = dscale_opt;
    r.gate_stride = a.gate_stride; r.scale_stride = a.scale_stride;
    r.B = s->B; r.chunks = a.chunks; r.C = s->C; r.w_f32 = a.w_f32; r.mod_f32 = a.mod_f32;
    CUDA_TRY(launch_dependent(blk::block_reduce_kernel, dim3(unsigned(ceil_div(s->C, 32))), dim3(32 * norm::kReduceWarps), 0, stream, r));
    count_launch();
    return CARNATOR_OK;
}

// ------------------------------------------------------------------------------------------------
// 8-bit operands
// ------------------------------------------------------------------------------------------------
namespace {
// Element strides of scales: those of axes longer than one are not negative and at most 2^38; `written`: values lie apart.
bool scales_ok(const int64_t* stride, const int64_t* size, int n, bool written) {
    int64_t st[3], sz[3], extent = 1;
    int used = 0;
    for (int i = 0; i < n; ++i) {
        if (size[i] == 1) continue;
        if (stride[i] < 0 || stride[i] > kMostStride) return false;
        st[used] = stride[i]; sz[used] = size[i]; ++used;
    }
    for (int k = 0; written && k < used; ++k) {
        int at = k;
        for (int i = k + 1; i < used; ++i) if (st[i] < st[at]) at = i;
        std::swap(st[k], st[at]); std::swap(sz[k], sz[at]);
        if (st[k] < extent) return false;
        extent += st[k] * (sz[k] - 1);
    }
    return true;
}
constexpr int64_t kMostAxis = int64_t(1) << 27;
}  // namespace

extern "C" carnator_status carnator_quantize_fp8(const void* X, const carnator_quantize_shape* s, void* Q, float* scale, void* stream_) {
    if (!s || s->B <= 0 || s->N <= 0 || s->K <= 0 || (s->block_rows != 1 && s->block_rows != fp8::kBlock) || !dtype_ok(s->x_dtype)) return CARNATOR_ERR_INVALID_ARG;
    const int blocks = ceil_div(s->K, fp8::kBlock), row_blocks = s->block_rows == 1 ? s->N : ceil_div(s->N, fp8::kBlock);
    if (int64_t(s->B) * s->N > kMostAxis || s->K > kMostAxis || s->B > 65535 || (s->block_rows > 1 && int64_t(row_blocks) * blocks > (int64_t(1) << 30))) return CARNATOR_ERR_UNSUPPORTED;
    if (!X || !Q || !scale || !aligned(X, 16) || !aligned(Q, 16) || !aligned(scale, 4)) return CARNATOR_ERR_INVALID_ARG;
    const int64_t size[2] = {s->B, s->N}, sizes[3] = {s->B, row_blocks, blocks};
    if (!axes_ok(s->x_stride, size, 2, s->K, s->x_dtype, false, false) || !axes_ok(s->q_stride, size, 2, s->K, CARNATOR_DTYPE_E4M3, true, false) ||
        !scales_ok(s->scale_stride, sizes, 3, true)) return CARNATOR_ERR_INVALID_ARG;
    const carnator_status st = check_device();
    if (st != CARNATOR_OK) return st;
    fp8::QuantArgs a = {};
    a.x = X; a.q = static_cast<uint8_t*>(Q); a.scale = scale;
    for (int i = 0; i < 2; ++i) { a.xs[i] = size[i] == 1 ? 0 : s->x_stride[i]; a.qs[i] = size[i] == 1 ? 0 : s->q_stride[i]; }
    for (int i = 0; i < 3; ++i) a.ss[i] = sizes[i] == 1 ? 0 : s->scale_stride[i];
    a.batches = s->B; a.rows = s->N; a.cols = s->K; a.blocks = blocks;
    const cudaError_t e = fp8::launch_quantize(a, s->x_dtype == CARNATOR_DTYPE_F32, s->block_rows, static_cast<cudaStream_t>(stream_));
    if (e != cudaSuccess) return cuda_fail(e, "quantize kernel");
    count_launch();
    return CARNATOR_OK;
}

namespace {
carnator_status check_fp8_shape(const carnator_linear_fp8_shape* s) {
    if (!s || s->B <= 0 || s->N <= 0 || s->in_features <= 0 || s->out_features <= 0) return CARNATOR_ERR_INVALID_ARG;
    if (s->activation < CARNATOR_ACT_NONE || s->activation > CARNATOR_ACT_SILU) return CARNATOR_ERR_INVALID_ARG;
    if ((!dtype_ok(s->x_dtype) && s->x_dtype != CARNATOR_DTYPE_E4M3) || !dtype_ok(s->y_dtype) || !dtype_ok(s->bias_dtype) || !dtype_ok(s->gate_dtype) || s->gate_stride < 0)
        return CARNATOR_ERR_INVALID_ARG;
    if (int64_t(s->B) * s->N > kMostAxis || s->in_features > kMostAxis || s->out_features > kMostAxis || s->B > 65535) return CARNATOR_ERR_UNSUPPORTED;
    return CARNATOR_OK;
}
bool few_rows(const carnator_linear_fp8_shape* s) { return int64_t(s->B) * s->N <= lin8::kRowsMost8; }

// Whether batch entries follow each other evenly, so that they are one run of rows.
bool entries_run(const carnator_linear_fp8_shape* s, const int64_t* stride) { return s->B == 1 || s->N == 1 || uint64_t(stride[0]) == uint64_t(s->N) * uint64_t(stride[1]); }
bool one_run(const carnator_linear_fp8_shape* s, bool residual) {
    return entries_run(s, s->x_stride) && entries_run(s, s->y_stride) && (!residual || entries_run(s, s->residual_stride)) &&
           (s->x_dtype != CARNATOR_DTYPE_E4M3 || entries_run(s, s->x_scale_stride));
}
// Status header, then what the two kernels of more than a few rows pass on; by the record alone: a call without a residual may take entries as one run that are not with it, which
// needs no more.
lin8::Room8 fp8_room(void* ws, const carnator_linear_fp8_shape* s) {
    const bool one = one_run(s, true);
    return lin8::room8_of(static_cast<char*>(ws) + align256(sizeof(WsHeader)), one ? 1 : s->B, one ? int64_t(s->B) * s->N : s->N, s->out_features, s->in_features,
                          s->x_dtype != CARNATOR_DTYPE_E4M3);
}
size_t fp8_ws_bytes(const carnator_linear_fp8_shape* s) { return align256(sizeof(WsHeader)) + (few_rows(s) ? 0 : fp8_room(nullptr, s).bytes); }
}  // namespace

extern "C" size_t carnator_linear_fp8_workspace_bytes(const carnator_linear_fp8_shape* s) {
    return check_fp8_shape(s) == CARNATOR_OK ? fp8_ws_bytes(s) : 0;
}

extern "C" carnator_status carnator_linear_fp8(const void* X, const float* x_scale, const void* W, const float* w_scale, const void* bias, const void* gate, const void* residual,
                                               const carnator_linear_fp8_shape* s, void* Y, void* ws, size_t ws_bytes, void* stream_) {
    carnator_status st = check_fp8_shape(s);
    if (st != CARNATOR_OK) return st;
    const bool ready = s->x_dtype == CARNATOR_DTYPE_E4M3;
    if (!X || !W || !w_scale || !Y || ready != (x_scale != nullptr)) return CARNATOR_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(Y, 16) || !aligned(residual, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4)) return CARNATOR_ERR_INVALID_ARG;
    if (!aligned(bias, size_t(dtype_bytes(s->bias_dtype))) || !aligned(gate, size_t(dtype_bytes(s->gate_dtype)))) return CARNATOR_ERR_INVALID_ARG;
    const int blocks = ceil_div(s->in_features, fp8::kBlock);
    const int64_t size[2] = {s->B, s->N}, xsize[3] = {s->B, s->N, blocks}, wsize[2] = {ceil_div(s->out_features, fp8::kBlock), blocks};
    auto rows_ok = [&](const int64_t* stride, int64_t row, int32_t dtype, bool written) { return axes_ok(stride, size, 2, row, dtype, written, true) && (s->N == 1 || stride[1] >= row); };
    if (!rows_ok(s->x_stride, s->in_features, s->x_dtype, false) || !rows_ok(s->y_stride, s->out_features, s->y_dtype, true) ||
        (residual && !rows_ok(s->residual_stride, s->out_features, s->y_dtype, false)) || (ready && !scales_ok(s->x_scale_stride, xsize, 3, false)) ||
        !scales_ok(s->w_scale_stride, wsize, 2, false)) return CARNATOR_ERR_INVALID_ARG;
    if (s->out_features > 1 && (s->w_stride < s->in_features || s->w_stride % 16 || s->w_stride > kMostStride)) return CARNATOR_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < fp8_ws_bytes(s)) return CARNATOR_ERR_WORKSPACE;
    st = check_device();
    if (st != CARNATOR_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    lin::Epilogue e = {};
    e.y = Y; e.bias = bias; e.gate = gate; e.residual = residual;
    // the stride of an axis of one entry may be anything
    int64_t xs[2], ys[2], rs[2], xss[3], wss[2];
    for (int i = 0; i < 2; ++i) {
        const bool one = size[i] == 1;
        xs[i] = one ? 0 : s->x_stride[i]; ys[i] = one ? 0 : s->y_stride[i]; rs[i] = one || !residual ? 0 : s->residual_stride[i];
        wss[i] = wsize[i] == 1 ? 0 : s->w_scale_stride[i];
    }
    for (int i = 0; i < 3; ++i) xss[i] = xsize[i] == 1 || !ready ? 0 : s->x_scale_stride[i];
    for (int i = 0; i < 2; ++i) { e.ys[i] = ys[i]; e.rs[i] = rs[i]; }
    e.gate_stride = s->B == 1 ? 0 : s->gate_stride;
    e.act = s->activation; e.y_f32 = s->y_dtype == CARNATOR_DTYPE_F32;
    e.bias_f32 = s->bias_dtype == CARNATOR_DTYPE_F32; e.gate_f32 = s->gate_dtype == CARNATOR_DTYPE_F32;
    e.vec_ok = vec16(bias, 0, s->bias_dtype) && vec16(gate, e.gate_stride, s->gate_dtype);
    e.wide_ok = rows32(Y, ys, s->y_dtype) && rows32(residual, rs, s->y_dtype);
    e.rows_per_gate = s->N;
    const int64_t rows = int64_t(s->B) * s->N;
    if (few_rows(s)) {
        lin8::RowsArgs8 a = {};
        a.e = e; a.x = X; a.w = static_cast<const uint8_t*>(W); a.xscale = x_scale; a.wscale = w_scale;
        for (int i = 0; i < 2; ++i) { a.xs[i] = xs[i]; a.wss[i] = wss[i]; }
        for (int i = 0; i < 3; ++i) a.xss[i] = xss[i];
        a.w_stride = s->out_features == 1 ? 0 : s->w_stride;
        a.hdr = static_cast<WsHeader*>(ws);
        a.rows = int(rows); a.per_batch = s->N; a.K = s->in_features; a.cols = s->out_features;
        const cudaError_t err = ready ? lin8::launch_rows8<lin8::kXE4m3>(a, stream)
                              : s->x_dtype == CARNATOR_DTYPE_F32 ? lin8::launch_rows8<lin8::kXF32>(a, stream) : lin8::launch_rows8<lin8::kXBf16>(a, stream);
        if (err != cudaSuccess) return cuda_fail(err, "linear_fp8_rows_kernel");
        count_launch();
        return CARNATOR_OK;
    }
    auto run_stride = [&](const int64_t* st) { return s->N == 1 ? st[0] : st[1]; };
    const lin8::Room8 room = fp8_room(ws, s);
    lin8::Args8 a = {};
    lin8::PrepareArgs p = {};
    a.t.e = e;
    a.t.hdr = static_cast<WsHeader*>(ws);
    a.wscale = p.wscale = w_scale;
    for (int i = 0; i < 2; ++i) a.wss[i] = p.wss[i] = wss[i];
    a.t.batches = s->B; a.t.rows = s->N;
    lin::Operand A = {X, s->B, s->N, s->in_features, xs[0], xs[1]};
    if (!ready) {
        p.q.x = X; p.q.q = room.q;
        p.q.xs[0] = xs[0]; p.q.xs[1] = xs[1];
        p.q.qs[0] = room.q_stride * s->N; p.q.qs[1] = room.q_stride;
        A.base = room.q; A.batch_stride = p.q.qs[0]; A.row_stride = p.q.qs[1];
    }
    if (one_run(s, residual != nullptr)) {
        a.t.batches = 1; a.t.rows = int(rows);
        A.batches = 1; A.rows = rows;
        if (ready) { A.row_stride = run_stride(xs); xss[1] = run_stride(xss); }
        else p.q.xs[1] = run_stride(xs);
        a.t.e.ys[1] = run_stride(ys); a.t.e.rs[1] = run_stride(rs);
    }
    a.xscale = p.xscale = x_scale;
    for (int i = 0; i < 3; ++i) a.xss[i] = p.xss[i] = xss[i];
    const lin::Operand Bo = {W, 1, s->out_features, s->in_features, 0, s->w_stride};
    a.t.cols = s->out_features;
    a.t.k_len = s->in_features;
    const int type = ready ? lin8::kXE4m3 : s->x_dtype == CARNATOR_DTYPE_F32 ? lin8::kXF32 : lin8::kXBf16;
    st = lin8::launch_product8(A, Bo, room, a, p, type, stream, g_cuda_error, sizeof(g_cuda_error));
    if (st == CARNATOR_OK) g_launches.fetch_add(2, std::memory_order_relaxed);
    return st;
}
