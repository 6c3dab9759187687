// C ABI of the operators around the attention call (layer norm, rotary positions, gradient of the Q/K preparation): argument checks.
#include <algorithm>
#include <cmath>

#include "clear_internal.hpp"

namespace {

using namespace clear;

bool misaligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }
size_t size_of(int dtype) { return dtype == CLEAR_BF16 ? 2 : 4; }
bool is_dtype(int dtype) { return dtype == CLEAR_BF16 || dtype == CLEAR_F32; }

// Launches' grids hold this many channels with room to spare.
constexpr int kMaxChannels = 1 << 23;

int check_norm(const NormArgs &a, const void *x, void *out)
{
    if (a.B < 0 || a.N < 0 || a.C <= 0 || !is_dtype(a.dtype) || !is_dtype(a.param_dtype)) return CLEAR_ERR_INVALID_ARG;
    if (a.dtype == CLEAR_F32 && a.param_dtype != CLEAR_F32) return CLEAR_ERR_INVALID_ARG;
    if (!(a.eps >= 0.f) || !std::isfinite(a.eps) || !std::isfinite(a.offset)) return CLEAR_ERR_INVALID_ARG;
    if ((long long)a.B * a.N > 0x7fffffffLL || a.C > kMaxChannels) return CLEAR_ERR_UNSUPPORTED;
    if (a.B == 0 || a.N == 0) return CLEAR_OK;
    if (!x || !out) return CLEAR_ERR_INVALID_ARG;
    // rows of the output that are one and the same
    if ((a.B > 1 && a.out_stride_b == 0) || (a.N > 1 && a.out_stride_n == 0)) return CLEAR_ERR_INVALID_ARG;
    const size_t e = size_of(a.dtype), pe = size_of(a.param_dtype);
    if (misaligned(x, e) || misaligned(out, e) || misaligned(a.weight, pe) || misaligned(a.bias, pe)) return CLEAR_ERR_MISALIGNED;
    if (misaligned(a.mean, 4) || misaligned(a.rstd, 4) || misaligned(a.mean_in, 4) || misaligned(a.rstd_in, 4))
        return CLEAR_ERR_MISALIGNED;
    return CLEAR_OK;
}

// The same strides, wherever an index reaches them.
bool same_rows(int B, int N, long long sb0, long long sn0, long long sb1, long long sn1)
{
    return (B <= 1 || sb0 == sb1) && (N <= 1 || sn0 == sn1);
}

int rope(const void *q, const void *k, void *q_out, void *k_out, const long long *strides, const void *positions,
         long long pos_stride_b, long long pos_stride_n, int position_bits, const double *frequencies, const int *axes_dim, int n_axes,
         int B, int H, int Hk, int N, int head_dim, int dtype, int layout, float factor, int inverse, void *stream)
{
    if (B < 0 || N < 0 || H <= 0 || head_dim <= 0 || n_axes <= 0 || !is_dtype(dtype)) return CLEAR_ERR_INVALID_ARG;
    if (layout != CLEAR_ROPE_INTERLEAVED && layout != CLEAR_ROPE_HALF) return CLEAR_ERR_INVALID_ARG;
    if (position_bits != 32 && position_bits != 64) return CLEAR_ERR_INVALID_ARG;
    if (!strides || !frequencies || !axes_dim || !std::isfinite(factor)) return CLEAR_ERR_INVALID_ARG;
    if ((k != nullptr) != (k_out != nullptr) || (k && Hk <= 0)) return CLEAR_ERR_INVALID_ARG;
    if (head_dim > 2 * kMaxRopePairs || n_axes > 8) return CLEAR_ERR_UNSUPPORTED;
    int rotary = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (axes_dim[a] < 0 || (axes_dim[a] & 1) || axes_dim[a] > head_dim - rotary) return CLEAR_ERR_INVALID_ARG;
        rotary += axes_dim[a];
    }
    if (rotary == 0) return CLEAR_ERR_INVALID_ARG;
    for (int p = 0; p < rotary / 2; ++p)
        if (!std::isfinite(frequencies[p])) return CLEAR_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return CLEAR_OK;
    if (!q || !q_out || !positions) return CLEAR_ERR_INVALID_ARG;
    RopeArgs a{};
    const void *in[2] = {q, k};
    void *out[2] = {q_out, k_out};
    const int heads[2] = {H, k ? Hk : 0};
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        const long long *s = strides + 6 * i, *o = s + 3;
        const int extent[3] = {B, heads[i], N};
        bool same = true;
        for (int d = 0; d < 3; ++d) {
            if (extent[d] > 1 && o[d] == 0) return CLEAR_ERR_INVALID_ARG;
            if (extent[d] > 1 && s[d] != o[d]) same = false;
        }
        if (in[i] == out[i] && !same) return CLEAR_ERR_INVALID_ARG;
        if (misaligned(in[i], size_of(dtype)) || misaligned(out[i], size_of(dtype))) return CLEAR_ERR_MISALIGNED;
        a.io[i] = RopeIo{in[i], out[i], heads[i], s[0], s[1], s[2], o[0], o[1], o[2]};
    }
    if (k && (q_out == k_out || q_out == k || k_out == q)) return CLEAR_ERR_INVALID_ARG;
    if (misaligned(positions, position_bits / 8)) return CLEAR_ERR_MISALIGNED;
    a.positions = positions;
    a.pos_stride_b = pos_stride_b;
    a.pos_stride_n = pos_stride_n;
    a.pos64 = position_bits == 64;
    a.frequencies = frequencies;
    a.axes_dim = axes_dim;
    a.n_axes = n_axes;
    a.B = B;
    a.N = N;
    a.head_dim = head_dim;
    a.dtype = dtype;
    a.half = layout == CLEAR_ROPE_HALF;
    a.inverse = inverse;
    a.factor = factor;
    return launch_rope(a, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

int clear_rope_frequencies(double *frequencies, int dim, double theta, int scaling, double factor, double trained_length, double fast,
                           double slow)
{
    if (!frequencies || dim <= 0 || (dim & 1)) return CLEAR_ERR_INVALID_ARG;
    if (!(theta > 0.) || !std::isfinite(theta) || !(factor > 0.) || !std::isfinite(factor)) return CLEAR_ERR_INVALID_ARG;
    if (scaling < CLEAR_ROPE_SCALE_NONE || scaling > CLEAR_ROPE_SCALE_PARTS) return CLEAR_ERR_INVALID_ARG;
    if (scaling == CLEAR_ROPE_SCALE_PARTS && (!(trained_length > 0.) || !std::isfinite(trained_length) || !std::isfinite(fast) ||
                                              !(slow >= 0.) || !(fast > slow)))
        return CLEAR_ERR_INVALID_ARG;
    if (scaling == CLEAR_ROPE_SCALE_NTK && dim > 2) theta *= std::pow(factor, (double)dim / (double)(dim - 2));
    for (int k = 0; k < dim / 2; ++k) {
        double w = std::pow(theta, -2.0 * (double)k / (double)dim);
        if (scaling == CLEAR_ROPE_SCALE_LINEAR) w /= factor;
        if (scaling == CLEAR_ROPE_SCALE_PARTS) {
            const double turns = trained_length * w / 6.283185307179586476925;
            const double keep = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            w *= keep + (1.0 - keep) / factor;
        }
        frequencies[k] = w;
    }
    return CLEAR_OK;
}

int clear_rope_fwd(const void *q, const void *k, void *q_out, void *k_out, const long long *strides, const void *positions,
                   long long pos_stride_b, long long pos_stride_n, int position_bits, const double *frequencies, const int *axes_dim,
                   int n_axes, int B, int H, int Hk, int N, int head_dim, int dtype, int layout, float factor, void *stream)
{
    return rope(q, k, q_out, k_out, strides, positions, pos_stride_b, pos_stride_n, position_bits, frequencies, axes_dim, n_axes, B, H,
                Hk, N, head_dim, dtype, layout, factor, 0, stream);
}

int clear_rope_bwd(const void *q, const void *k, void *q_out, void *k_out, const long long *strides, const void *positions,
                   long long pos_stride_b, long long pos_stride_n, int position_bits, const double *frequencies, const int *axes_dim,
                   int n_axes, int B, int H, int Hk, int N, int head_dim, int dtype, int layout, float factor, void *stream)
{
    return rope(q, k, q_out, k_out, strides, positions, pos_stride_b, pos_stride_n, position_bits, frequencies, axes_dim, n_axes, B, H,
                Hk, N, head_dim, dtype, layout, factor, 1, stream);
}

int clear_layer_norm_fwd(const void *x, void *y, const void *weight, const void *bias, float *mean, float *rstd, int B, int N, int C,
                         int dtype, int param_dtype, long long x_stride_b, long long x_stride_n, long long y_stride_b,
                         long long y_stride_n, long long weight_stride_b, long long bias_stride_b, float weight_offset, float eps,
                         void *stream)
{
    NormArgs a{};
    a.x = x; a.out = y; a.weight = weight; a.bias = bias; a.mean = mean; a.rstd = rstd;
    a.B = B; a.N = N; a.C = C; a.dtype = dtype; a.param_dtype = param_dtype;
    a.x_stride_b = x_stride_b; a.x_stride_n = x_stride_n; a.out_stride_b = y_stride_b; a.out_stride_n = y_stride_n;
    a.w_stride_b = weight_stride_b; a.bias_stride_b = bias_stride_b;
    a.offset = weight_offset; a.eps = eps;
    const int rc = check_norm(a, x, y);
    if (rc != CLEAR_OK || B == 0 || N == 0) return rc;
    if (x == y && !same_rows(B, N, x_stride_b, x_stride_n, y_stride_b, y_stride_n)) return CLEAR_ERR_INVALID_ARG;
    return launch_norm_fwd(a, static_cast<cudaStream_t>(stream));
}

int clear_layer_norm_bwd_workspace(int B, int N, int C, int per_batch, size_t *bytes)
{
    if (!bytes || B < 0 || N < 0 || C <= 0) return CLEAR_ERR_INVALID_ARG;
    if ((long long)B * N > 0x7fffffffLL || C > kMaxChannels || (per_batch && B > 65535)) return CLEAR_ERR_UNSUPPORTED;
    *bytes = 0;
    return B == 0 || N == 0 ? CLEAR_OK : norm_bwd_workspace(B, N, C, per_batch != 0, bytes);
}

int clear_layer_norm_bwd(const void *x, const void *dy, const void *weight, const float *mean, const float *rstd, void *dx,
                         void *dweight, void *dbias, int B, int N, int C, int dtype, int param_dtype, int per_batch,
                         long long x_stride_b, long long x_stride_n, long long dy_stride_b, long long dy_stride_n,
                         long long dx_stride_b, long long dx_stride_n, long long weight_stride_b, long long dweight_stride_b,
                         long long dbias_stride_b, float weight_offset, void *workspace, size_t workspace_bytes, void *stream)
{
    NormArgs a{};
    a.x = x; a.dy = dy; a.out = dx; a.weight = weight; a.dweight = dweight; a.dbias = dbias;
    a.mean_in = mean; a.rstd_in = rstd;
    a.B = B; a.N = N; a.C = C; a.dtype = dtype; a.param_dtype = param_dtype; a.per_batch = per_batch != 0;
    a.x_stride_b = x_stride_b; a.x_stride_n = x_stride_n; a.dy_stride_b = dy_stride_b; a.dy_stride_n = dy_stride_n;
    a.out_stride_b = dx_stride_b; a.out_stride_n = dx_stride_n;
    a.w_stride_b = weight_stride_b; a.dw_stride_b = dweight_stride_b; a.db_stride_b = dbias_stride_b;
    a.offset = weight_offset;
    a.workspace = workspace;
    const int rc = check_norm(a, x, dx);
    if (rc != CLEAR_OK) return rc;
    if (misaligned(dweight, size_of(param_dtype)) || misaligned(dbias, size_of(param_dtype))) return CLEAR_ERR_MISALIGNED;
    if (per_batch) {
        if (B > 65535) return CLEAR_ERR_UNSUPPORTED;
        if (B > 1 && ((dweight && dweight_stride_b == 0) || (dbias && dbias_stride_b == 0))) return CLEAR_ERR_INVALID_ARG;
    } else if ((weight && weight_stride_b) || (dweight && dweight_stride_b) || (dbias && dbias_stride_b)) {
        return CLEAR_ERR_INVALID_ARG;
    }
    if (dweight && dweight == dbias) return CLEAR_ERR_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0 || N == 0) {
        const size_t width = (size_t)C * size_of(param_dtype);
        for (int i = 0; i < 2; ++i) {
            void *sum = i == 0 ? dweight : dbias;
            const long long stride = i == 0 ? dweight_stride_b : dbias_stride_b;
            for (int b = 0; sum && b < (per_batch ? B : 1); ++b)
                CLEAR_CUDA_TRY(cudaMemsetAsync(static_cast<char *>(sum) + (long long)b * stride * (long long)size_of(param_dtype), 0,
                                               width, s));
        }
        return CLEAR_OK;
    }
    if (!dy || !mean || !rstd) return CLEAR_ERR_INVALID_ARG;
    if (misaligned(dy, size_of(dtype))) return CLEAR_ERR_MISALIGNED;
    if ((dx == x && !same_rows(B, N, x_stride_b, x_stride_n, dx_stride_b, dx_stride_n)) ||
        (dx == dy && !same_rows(B, N, dy_stride_b, dy_stride_n, dx_stride_b, dx_stride_n)))
        return CLEAR_ERR_INVALID_ARG;
    if (dweight || dbias) {
        size_t need = 0;
        if (const int e = norm_bwd_workspace(B, N, C, a.per_batch, &need)) return e;
        if (need && (!workspace || workspace_bytes < need)) return CLEAR_ERR_INVALID_ARG;
        if (misaligned(workspace, 16)) return CLEAR_ERR_MISALIGNED;
    }
    return launch_norm_bwd(a, s);
}

int clear_qk_norm_rope_bwd_workspace(int head_dim, size_t *bytes)
{
    if (!bytes || head_dim <= 0) return CLEAR_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return CLEAR_ERR_UNSUPPORTED;
    return prep_bwd_workspace(head_dim, bytes);
}

int clear_qk_norm_rope_bwd(const void *q, const void *k, const void *dq_rot, const void *dk_rot, void *dq, void *dk,
                           const float *gain_q, const float *gain_k, float *dgain_q, float *dgain_k, int B, int H, int grid_h,
                           int grid_w, int n_text, int head_dim, int dtype, int axis0_dim, int axis1_dim, int axis2_dim, float theta,
                           float ntk_factor, float eps, float q_factor, void *workspace, size_t workspace_bytes, void *stream)
{
    if (B <= 0 || H <= 0 || grid_h <= 0 || grid_w <= 0 || n_text < 0 || !is_dtype(dtype)) return CLEAR_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return CLEAR_ERR_UNSUPPORTED;
    const int axes[3] = {axis0_dim, axis1_dim, axis2_dim};
    for (int dim : axes)
        if (dim < 0 || (dim & 1)) return CLEAR_ERR_INVALID_ARG;
    if ((long long)axis0_dim + axis1_dim + axis2_dim != head_dim) return CLEAR_ERR_INVALID_ARG;
    if (!(theta > 0.f) || !std::isfinite(theta) || !(ntk_factor > 0.f) || !std::isfinite(ntk_factor)) return CLEAR_ERR_INVALID_ARG;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(q_factor)) return CLEAR_ERR_INVALID_ARG;
    for (const void *p : {q, k, dq_rot, dk_rot, (const void *)dq, (const void *)dk}) {
        if (!p) return CLEAR_ERR_INVALID_ARG;
        if (misaligned(p, 16)) return CLEAR_ERR_MISALIGNED;
    }
    if (dq == dk || dq == k || dq == dk_rot || dk == q || dk == dq_rot) return CLEAR_ERR_INVALID_ARG;
    if (misaligned(gain_q, 4) || misaligned(gain_k, 4) || misaligned(dgain_q, 4) || misaligned(dgain_k, 4)) return CLEAR_ERR_MISALIGNED;
    if ((long long)B * H > 0x7fffffffLL || n_text + (long long)grid_h * grid_w > 0x7fffffffLL) return CLEAR_ERR_UNSUPPORTED;
    if (dgain_q || dgain_k) {
        if (dgain_q == dgain_k) return CLEAR_ERR_INVALID_ARG;
        size_t need = 0;
        if (const int rc = prep_bwd_workspace(head_dim, &need)) return rc;
        if (!workspace || workspace_bytes < need) return CLEAR_ERR_INVALID_ARG;
        if (misaligned(workspace, 16)) return CLEAR_ERR_MISALIGNED;
    }
    return launch_prep_bwd(q, k, dq_rot, dk_rot, dq, dk, gain_q, gain_k, dgain_q, dgain_k, B * H, grid_h, grid_w, n_text, head_dim, dtype,
                           axes, (double)theta, (double)ntk_factor, eps, q_factor, workspace, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
