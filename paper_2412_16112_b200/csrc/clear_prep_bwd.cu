// Gradient of the Q/K preparation (clear_prep.cu): y = f R(t) (x inv gain), inv = 1 / sqrt(mean(x^2) + eps), per row of Q and of K.
//
//   u = f R(-t) dy,   s = u gain,   dx = inv (s - x inv^2 mean(s x)),   dgain = sum over all rows of u x inv
//
// HBM bounds it: x and dy in once, dx out once.  As in the forward kernel a thread owns 8 channels of a token and walks over its
// (batch, head) rows, so sines and cosines are computed once a token; the gains' gradients stay in its registers all the while.
// Device time, and bytes over the measured copy rate of 6541 GB/s: 4096 px bf16 382 to 412 us by where the tensors
// lie, 0.90 to 0.97; 1024 px bf16 32.0 us, 0.81 (4 us of it
// the second kernel, which adds the blocks' sums of the gains' gradients), fp32 58 us, 0.90; the tiny fp32 shape 6.3 us.
// 135 warp instructions for a warp's row of 8 channels a lane; fewer of them also means a higher clock under the board's power cap.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "clear_internal.hpp"
#include "launch_once.hpp"
#include "ptx.cuh"
#include "rope_angle.cuh"
#include "row_io.cuh"

namespace clear {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kEpl = 8;  // channels a thread
constexpr int kBlocksPerSm = 2;

struct PrepBwdParams {
    const void *x[2], *dy[2];
    void *dx[2];
    const float *gain[2];
    float *partial;             // [blocks][2][d], or null
    float *dgain[2];            // without partial sums: where the one cluster of blocks writes its sums itself
    int n_bh, bh_a_part;        // rows of a token, and of the shares that blocks take of them
    unsigned parts, n_text, grid_w, n_tokens;
    float eps, factor[2];
    uint64_t turns[64];
    uint8_t axis[64];
};

// Rows come ahead by asynchronous copies of each thread's own channels into its own places of shared memory (bf16: 16 bytes, two
// steps of three rows, 385 us at 4096 px where three rows ahead in registers take 410), or in registers where 8 channels are two
// accesses (fp32, 4608 tokens of 24 heads, two rows: 58 us, copies 91).
template <typename T> constexpr bool kAhead = sizeof(T) == 2;
template <typename T> constexpr int kRowsOf = kAhead<T> ? 3 : 2;
template <typename T> constexpr int kRingBytes = kAhead<T> ? 2 * kRowsOf<T> * 2 * kThreads * 16 : 0;

// Even warps have rows of Q, odd ones rows of K, so that a thread keeps one gain and one gain's gradient.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) clear_prep_bwd_kernel(const __grid_constant__ PrepBwdParams p)
{
    constexpr int kLanes = D / kEpl, kTokens = 32 / kLanes, kPairs = kEpl / 2, kRows = kRowsOf<T>;
    extern __shared__ __align__(16) unsigned char s_ring[];  // two steps: [kRows][x, dy][kThreads][16]
    __shared__ float s_gain[kWarps][kTokens][D], s_sum[2 * D];
    __shared__ uint64_t s_turns[D / 2];
    __shared__ uint8_t s_axis[D / 2];
    for (int i = threadIdx.x; i < D / 2; i += kThreads) {
        s_turns[i] = p.turns[i];
        s_axis[i] = p.axis[i];
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, c0 = (lane % kLanes) * kEpl;
    const int w = warp & 1;
    const T *x_in = static_cast<const T *>(p.x[w]), *dy_in = static_cast<const T *>(p.dy[w]);
    T *dx_out = static_cast<T *>(p.dx[w]);
    const float factor = p.factor[w];
    F2 gain[kPairs], dgain[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        gain[i] = p.gain[w] ? F2(__ldg(p.gain[w] + c0 + 2 * i), __ldg(p.gain[w] + c0 + 2 * i + 1)) : F2(1.f);
        dgain[i] = F2(0.f);
    }
    const long long stride = (long long)p.n_tokens * D;
    const uint32_t ring = ptx::smem_u32(s_ring) + threadIdx.x * 16;
    const unsigned jobs = (p.n_tokens + kTokens - 1) / kTokens * p.parts;
    for (unsigned job = blockIdx.x * (kWarps / 2) + warp / 2; job < jobs; job += gridDim.x * (kWarps / 2)) {
        const unsigned grp = job / p.parts, raw = grp * kTokens + sub;
        const int bh0 = (int)(job - grp * p.parts) * p.bh_a_part, bh1 = min(p.n_bh, bh0 + p.bh_a_part);
        const bool live = raw < p.n_tokens;
        const unsigned n = live ? raw : p.n_tokens - 1;  // the lanes stay together for the shuffles; what they add does not count
        const long long elem = (long long)n * D + c0;
        Pack<T, kEpl> nx[kRows], nd[kRows];
        constexpr uint32_t kSlot = kThreads * 16, kStage = kRows * 2 * kSlot;
        const T *x_at = x_in + elem + bh0 * stride, *dy_at = dy_in + elem + bh0 * stride;
        T *dx_at = dx_out + elem + bh0 * stride;
        int ahead = bh0;
        auto fetch = [&](uint32_t to) {  // the next kRows rows, into a stage (by its offset in bytes)
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const bool there = ahead + j < bh1;
                if constexpr (kAhead<T>) {
                    copy_async_if(ring + to + 2 * j * kSlot, x_at, there);
                    copy_async_if(ring + to + (2 * j + 1) * kSlot, dy_at, there);
                } else if (there) {
                    nx[j].load(x_at);
                    nd[j].load(dy_at);
                }
                x_at += stride;
                dy_at += stride;
            }
            ahead += kRows;
            if constexpr (kAhead<T>) copies_commit();
        };
        fetch(0);
        int pos[3] = {0, 0, 0};
        if (n >= p.n_text) {
            pos[1] = (int)((n - p.n_text) / p.grid_w);
            pos[2] = (int)(n - p.n_text) - pos[1] * (int)p.grid_w;
        }
        float sn[kPairs], cs[kPairs];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const int axis = s_axis[c0 / 2 + i];
            turn_sincos(axis == 1 ? pos[1] : axis == 2 ? pos[2] : 0, s_turns[c0 / 2 + i], sn[i], cs[i]);
            sn[i] *= factor;
            cs[i] *= factor;
        }
        uint32_t stage = 0;
        for (int bh = bh0; bh < bh1; bh += kRows) {
            if constexpr (kAhead<T>) {
                fetch(stage ^ kStage);
                copies_wait<1>();
            }
            F2 x2[kRows][kPairs], u2[kRows][kPairs];
            float ss[kRows], sx[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                if constexpr (kAhead<T>) {  // beyond the last row: what lies there is not used
                    const unsigned char *at = s_ring + stage + 2 * j * kSlot + threadIdx.x * 16;
                    nx[j].load(reinterpret_cast<const T *>(at));
                    nd[j].load(reinterpret_cast<const T *>(at + kSlot));
                }
                float x[kEpl], u[kEpl];
                nx[j].get(x);
                nd[j].get(u);
                F2 squares(0.f), products(0.f);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float a = u[2 * i], b = u[2 * i + 1];
                    u2[j][i] = F2(fmaf(b, sn[i], a * cs[i]), fmaf(-a, sn[i], b * cs[i]));
                    x2[j][i] = F2(x[2 * i], x[2 * i + 1]);
                    squares = fma2(x2[j][i], x2[j][i], squares);
                    products = fma2(u2[j][i] * gain[i], x2[j][i], products);
                }
                ss[j] = squares.lo() + squares.hi();
                sx[j] = products.lo() + products.hi();
            }
            stage ^= kStage;
            if constexpr (!kAhead<T>) fetch(0);
            // half of a row's lanes add up its squares, the others its products, and they swap
            const bool second = lane & (kLanes / 2);
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                float mine = second ? sx[j] : ss[j];
                mine += __shfl_xor_sync(0xffffffffu, second ? ss[j] : sx[j], kLanes / 2);
#pragma unroll
                for (int off = kLanes / 4; off > 0; off >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, off);
                const float other = __shfl_xor_sync(0xffffffffu, mine, kLanes / 2);
                ss[j] = second ? other : mine;
                sx[j] = second ? mine : other;
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                if (bh + j < bh1 && live) {
                    const float inv = rsqrtf(fmaf(ss[j], 1.f / D, p.eps));
                    const F2 inv2(inv), along(-(sx[j] * inv) * (1.f / D) * inv * inv);  // in an order that stays in range
                    float o[kEpl];
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        const F2 ui = u2[j][i] * inv2;
                        dgain[i] = fma2(ui, x2[j][i], dgain[i]);
                        const F2 r = fma2(x2[j][i], along, ui * gain[i]);
                        o[2 * i] = r.lo();
                        o[2 * i + 1] = r.hi();
                    }
                    Pack<T, kEpl> out;
                    out.set(o);
                    out.store(dx_at);
                }
                dx_at += stride;
            }
        }
        if constexpr (kAhead<T>) copies_wait<0>();
    }
    if (!p.partial && !p.dgain[0] && !p.dgain[1]) return;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        s_gain[warp][sub][c0 + 2 * i] = dgain[i].lo();
        s_gain[warp][sub][c0 + 2 * i + 1] = dgain[i].hi();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps / 2 * kTokens; ++k) sum += s_gain[2 * (k / kTokens) + i / D][k % kTokens][i % D];
        if (p.partial) p.partial[(size_t)blockIdx.x * 2 * D + i] = sum;
        else s_sum[i] = sum;
    }
    if (p.partial) return;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();  // the blocks' sums, each in its own shared memory
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < 2 * D; i += gridDim.x * kThreads) {
        float sum = 0.f;
        for (int k = 0; k < (int)gridDim.x; ++k) sum += cluster.map_shared_rank(s_sum, k)[i];
        if (p.dgain[i / D]) p.dgain[i / D][i % D] = sum;
    }
    cluster.sync();  // nobody leaves while its sums are read
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

template <typename T, int D>
int launch(PrepBwdParams &p, float *dgain_q, float *dgain_k, int device, int most, cudaStream_t stream)
{
    constexpr int kTokens = 32 / (D / kEpl);
    const int groups = (int)((p.n_tokens + kTokens - 1) / kTokens);
    // Few rows go to one cluster of blocks that adds up its sums itself: the host, which small calls wait for, has one launch instead of
    // two (20 us for 24), and the device is done sooner (20 tokens of 2 heads of 64: 4.1 and 4.8 us) or somewhat later (272: 6.5 and 4.6).
    const bool direct = p.partial && (long long)p.n_bh * p.n_tokens * D <= 48 * 1024;
    if (direct) {
        most = 8;
        p.partial = nullptr;
        p.dgain[0] = dgain_q;
        p.dgain[1] = dgain_k;
    }
    // the rows of a token are shared out while tokens alone leave warps without work
    const int warps = most * (kWarps / 2), parts = std::min(p.n_bh, std::max(1, warps / groups));
    p.bh_a_part = (p.n_bh + parts - 1) / parts;
    p.parts = (unsigned)((p.n_bh + p.bh_a_part - 1) / p.bh_a_part);
    int blocks = (int)std::min<long long>(most, ((long long)groups * p.parts + kWarps / 2 - 1) / (kWarps / 2));
    if (direct)
        while (blocks & (blocks - 1)) ++blocks;  // 1, 2, 4 or 8
    constexpr int smem = kRingBytes<T>;
    static std::atomic<int> known[kMaxDevices];
    int per_sm = 0;
    if (const int rc = kernel_once(known, clear_prep_bwd_kernel<T, D>, kThreads, smem, device, &per_sm)) return rc;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = direct && blocks > 1;
    CLEAR_CUDA_TRY(cudaLaunchKernelEx(&cfg, clear_prep_bwd_kernel<T, D>, p));
    if (!p.partial) return CLEAR_OK;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * D / 8);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    CLEAR_CUDA_TRY(cudaLaunchKernelEx(&cfg, clear_prep_gain_kernel<D>, (const float *)p.partial, blocks, dgain_q, dgain_k));
    return CLEAR_OK;
}

}  // namespace

int prep_bwd_workspace(int head_dim, size_t *bytes)
{
    int device = 0, n_sm = 0;
    if (const int rc = current_sms(&device, &n_sm)) return rc;
    *bytes = (size_t)kBlocksPerSm * n_sm * 2 * head_dim * sizeof(float);
    return CLEAR_OK;
}

int launch_prep_bwd(const void *q, const void *k, const void *dq_rot, const void *dk_rot, void *dq, void *dk, const float *gain_q,
                    const float *gain_k, float *dgain_q, float *dgain_k, int n_bh, int grid_h, int grid_w, int n_text, int head_dim,
                    int dtype, const int axes_dim[3], double theta, double ntk_factor, float eps, float q_factor, void *workspace,
                    cudaStream_t stream)
{
    int device = 0, n_sm = 0;
    if (const int rc = current_sms(&device, &n_sm)) return rc;
    const int most = kBlocksPerSm * n_sm;
    PrepBwdParams p{};
    p.x[0] = q; p.x[1] = k;
    p.dy[0] = dq_rot; p.dy[1] = dk_rot;
    p.dx[0] = dq; p.dx[1] = dk;
    p.gain[0] = gain_q; p.gain[1] = gain_k;
    p.partial = dgain_q || dgain_k ? static_cast<float *>(workspace) : nullptr;
    p.n_bh = n_bh;
    p.n_text = (unsigned)n_text;
    p.grid_w = (unsigned)grid_w;
    p.n_tokens = (unsigned)(n_text + (long long)grid_h * grid_w);
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
        return head_dim == 128 ? launch<__nv_bfloat16, 128>(p, dgain_q, dgain_k, device, most, stream)
                               : launch<__nv_bfloat16, 64>(p, dgain_q, dgain_k, device, most, stream);
    return head_dim == 128 ? launch<float, 128>(p, dgain_q, dgain_k, device, most, stream)
                           : launch<float, 64>(p, dgain_q, dgain_k, device, most, stream);
}

}  // namespace clear
