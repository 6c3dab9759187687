// Gradient of the Q/K preparation (clear_prep.cu): y = f R(t) (x inv gain), inv = 1 / sqrt(mean(x^2) + eps), per row of Q and of K.
//
//   u = f R(-t) dy,   s = u gain,   dx = inv (s - x inv^2 mean(s x)),   dgain = sum over all rows of u x inv
//
// HBM bounds it: x and dy in once, dx out once.  As in the forward kernel a thread owns 8 channels of a token and walks over its
// (batch, head) rows, so sines and cosines are computed once a token; the gains' gradients stay in its registers all the while.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "clear_internal.hpp"
#include "ptx.cuh"
#include "rope_angle.cuh"
#include "row_io.cuh"

namespace clear {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kEpl = 8;  // channels a thread

struct PrepBwdParams {
    const void *x[2], *dy[2];
    void *dx[2];
    const float *gain[2];
    float *partial;             // [blocks][2][d], or null
    int n_bh, bh_a_part, parts; // rows of a token, and the shares that blocks take of them
    int n_text, grid_w;
    long long n_tokens;
    float eps, factor[2];
    uint64_t turns[64];
    uint8_t axis[64];
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) clear_prep_bwd_kernel(const __grid_constant__ PrepBwdParams p)
{
    constexpr int kLanes = D / kEpl, kTokens = 32 / kLanes, kRows = 2;
    __shared__ float s_gain[kWarps][kTokens][2][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, c0 = (lane % kLanes) * kEpl;
    float gain[2][kEpl], dgain[2][kEpl];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < kEpl; ++i) {
            gain[w][i] = p.gain[w] ? __ldg(p.gain[w] + c0 + i) : 1.f;
            dgain[w][i] = 0.f;
        }
    const long long stride = p.n_tokens * D, groups = (p.n_tokens + kTokens - 1) / kTokens;
    for (long long job = (long long)blockIdx.x * kWarps + warp; job < groups * p.parts; job += (long long)gridDim.x * kWarps) {
        const long long grp = job / p.parts;
        const int bh0 = (int)(job - grp * p.parts) * p.bh_a_part, bh1 = min(p.n_bh, bh0 + p.bh_a_part);
        const long long raw = grp * kTokens + sub;
        const bool live = raw < p.n_tokens;
        const long long n = live ? raw : p.n_tokens - 1;  // the lanes stay together for the shuffles; what they add does not count
        int pos[3] = {0, 0, 0};
        if (n >= p.n_text) {
            const long long at = n - p.n_text;
            pos[1] = (int)(at / p.grid_w);
            pos[2] = (int)(at - (long long)pos[1] * p.grid_w);
        }
        float sn[kEpl / 2], cs[kEpl / 2];
#pragma unroll
        for (int i = 0; i < kEpl / 2; ++i) {
            const int axis = p.axis[c0 / 2 + i];
            turn_sincos(axis == 1 ? pos[1] : axis == 2 ? pos[2] : 0, p.turns[c0 / 2 + i], sn[i], cs[i]);
        }
        const long long elem = n * D + c0;
        auto row = [&](auto which, const Pack<T, kEpl> &rx, const Pack<T, kEpl> &rd, long long at) {
            constexpr int w = decltype(which)::value;
            float x[kEpl], u[kEpl];
            rx.get(x);
            rd.get(u);
            float ss = 0.f, sx = 0.f;
#pragma unroll
            for (int i = 0; i < kEpl / 2; ++i) {
                const float a = u[2 * i] * p.factor[w], b = u[2 * i + 1] * p.factor[w];
                u[2 * i] = a * cs[i] + b * sn[i];
                u[2 * i + 1] = b * cs[i] - a * sn[i];
            }
#pragma unroll
            for (int i = 0; i < kEpl; ++i) {
                ss = fmaf(x[i], x[i], ss);
                sx = fmaf(u[i] * gain[w][i], x[i], sx);
            }
#pragma unroll
            for (int off = kLanes / 2; off > 0; off >>= 1) {
                ss += __shfl_xor_sync(0xffffffffu, ss, off);
                sx += __shfl_xor_sync(0xffffffffu, sx, off);
            }
            const float inv = rsqrtf(fmaf(ss, 1.f / D, p.eps)), along = sx * (1.f / D) * inv * inv;
            if (live) {
                Pack<T, kEpl> out;
#pragma unroll
                for (int i = 0; i < kEpl; ++i) {
                    dgain[w][i] = fmaf(u[i], x[i] * inv, dgain[w][i]);
                    u[i] = inv * (u[i] * gain[w][i] - x[i] * along);
                }
                out.set(u);
                out.store(static_cast<T *>(p.dx[w]) + at);
            }
        };
        for (int bh = bh0; bh < bh1; bh += kRows) {
            Pack<T, kEpl> rx[2][kRows], rd[2][kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const long long at = elem + (long long)min(bh + j, bh1 - 1) * stride;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    rx[w][j].load(static_cast<const T *>(p.x[w]) + at);
                    rd[w][j].load(static_cast<const T *>(p.dy[w]) + at);
                }
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                if (bh + j < bh1) {
                    const long long at = elem + (long long)(bh + j) * stride;
                    row(std::integral_constant<int, 0>{}, rx[0][j], rd[0][j], at);
                    row(std::integral_constant<int, 1>{}, rx[1][j], rd[1][j], at);
                }
            }
        }
    }
    if (!p.partial) return;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < kEpl; ++i) s_gain[warp][sub][w][c0 + i] = dgain[w][i];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps * kTokens; ++k) sum += s_gain[k / kTokens][k % kTokens][i / D][i % D];
        p.partial[(size_t)blockIdx.x * 2 * D + i] = sum;
    }
}

// A warp to a channel of a gain: sums of the blocks' partial sums in a fixed order.
template <int D>
__global__ void __launch_bounds__(256) clear_prep_gain_kernel(const float *partial, int parts, float *dgain_q, float *dgain_k)
{
    ptx::grid_wait();
    const int col = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    float sum = 0.f;
    for (int i = lane; i < parts; i += 32) sum += partial[(size_t)i * 2 * D + col];
    sum = warp_sum(sum);
    float *out = col < D ? dgain_q : dgain_k;
    if (lane == 0 && out) out[col % D] = sum;
}

int grid_size(int *blocks)
{
    int dev = 0, n_sm = 0;
    CLEAR_CUDA_TRY(cudaGetDevice(&dev));
    CLEAR_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
    *blocks = 2 * n_sm;
    return CLEAR_OK;
}

template <typename T, int D>
int launch(PrepBwdParams &p, float *dgain_q, float *dgain_k, int most, cudaStream_t stream)
{
    constexpr int kTokens = 32 / (D / kEpl);
    const long long groups = (p.n_tokens + kTokens - 1) / kTokens, warps = (long long)most * kWarps;
    // the rows of a token are shared out while tokens alone leave warps without work
    p.parts = (int)std::min<long long>(p.n_bh, std::max<long long>(1, warps / groups));
    p.bh_a_part = (p.n_bh + p.parts - 1) / p.parts;
    p.parts = (p.n_bh + p.bh_a_part - 1) / p.bh_a_part;
    const int blocks = (int)std::min<long long>(most, (groups * p.parts + kWarps - 1) / kWarps);
    clear_prep_bwd_kernel<T, D><<<blocks, kThreads, 0, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    if (!p.partial) return CLEAR_OK;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * D / 8);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    CLEAR_CUDA_TRY(cudaLaunchKernelEx(&cfg, clear_prep_gain_kernel<D>, (const float *)p.partial, blocks, dgain_q, dgain_k));
    return CLEAR_OK;
}

}  // namespace

int prep_bwd_workspace(int head_dim, size_t *bytes)
{
    int blocks = 0;
    if (const int rc = grid_size(&blocks)) return rc;
    *bytes = (size_t)blocks * 2 * head_dim * sizeof(float);
    return CLEAR_OK;
}

int launch_prep_bwd(const void *q, const void *k, const void *dq_rot, const void *dk_rot, void *dq, void *dk, const float *gain_q,
                    const float *gain_k, float *dgain_q, float *dgain_k, int n_bh, int grid_h, int grid_w, int n_text, int head_dim,
                    int dtype, const int axes_dim[3], double theta, double ntk_factor, float eps, float q_factor, void *workspace,
                    cudaStream_t stream)
{
    int most = 0;
    if (const int rc = grid_size(&most)) return rc;
    PrepBwdParams p{};
    p.x[0] = q; p.x[1] = k;
    p.dy[0] = dq_rot; p.dy[1] = dk_rot;
    p.dx[0] = dq; p.dx[1] = dk;
    p.gain[0] = gain_q; p.gain[1] = gain_k;
    p.partial = dgain_q || dgain_k ? static_cast<float *>(workspace) : nullptr;
    p.n_bh = n_bh;
    p.n_text = n_text;
    p.grid_w = grid_w;
    p.n_tokens = (long long)n_text + (long long)grid_h * grid_w;
    p.eps = eps;
    p.factor[0] = q_factor;
    p.factor[1] = 1.f;
    int pair = 0;
    for (int a = 0; a < 3; ++a) {
        const int dim = axes_dim[a];
        double base = theta;
        if (dim > 2) base *= std::pow(ntk_factor, (double)dim / (double)(dim - 2));
        for (int i = 0; i < dim / 2; ++i, ++pair) {
            p.turns[pair] = turns_of(std::pow(base, -2.0 * (double)i / (double)dim));
            p.axis[pair] = (uint8_t)a;
        }
    }
    if (dtype == CLEAR_BF16)
        return head_dim == 128 ? launch<__nv_bfloat16, 128>(p, dgain_q, dgain_k, most, stream)
                               : launch<__nv_bfloat16, 64>(p, dgain_q, dgain_k, most, stream);
    return head_dim == 128 ? launch<float, 128>(p, dgain_q, dgain_k, most, stream)
                           : launch<float, 64>(p, dgain_q, dgain_k, most, stream);
}

}  // namespace clear
