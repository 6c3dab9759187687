// Layer normalisation of rows of C channels, forward and backward, with a gain and a bias that all rows share or that each batch
// entry has of its own (a diffusion transformer's modulation: gain 1 + scale, bias shift).
//
//   h = (x - mean) rstd,   y = h G + bias,   G = weight_offset + weight
//   g = dy G,   dx = rstd (g - mean(g) - h mean(g h)),   dweight = sum of dy h over the rows,   dbias = sum of dy
//
// HBM bounds all of it: x once in and y once out, or x and dy in and dx out, so a row stays in registers between its two uses.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "clear_internal.hpp"
#include "ptx.cuh"
#include "row_io.cuh"

namespace clear {
namespace {

constexpr int kMaxRowWarps = 16;

struct NormParams {
    const void *x, *dy;
    void *out;                    // y, or dx
    const void *weight, *bias;
    const float *mean_in, *rstd_in;
    float *mean, *rstd;
    float *partial;               // backward: [groups][blocks of a group][2][C]
    long long x_stride_b, x_stride_n, dy_stride_b, dy_stride_n, out_stride_b, out_stride_n;
    long long w_stride_b, bias_stride_b;
    unsigned rows, n_rows_b;      // all rows, rows of a batch entry
    int C, n_vec;                 // channels, accesses of V channels a row
    int row_warps, groups;        // warps that share a row, rows a block has in work at a time
    int per_batch;                // backward: gradients of the weights for each batch entry
    float offset, eps;
};

// Merge of the row_warps warps' (sum-like) values: every lane of every warp gets the totals.
struct RowGroup {
    int warp, lane, grp, row_warps;
    __device__ __forceinline__ RowGroup(int rw)
        : warp((threadIdx.x >> 5) % rw), lane(threadIdx.x & 31), grp((threadIdx.x >> 5) / rw), row_warps(rw)
    {
    }
};

// ---- forward ---------------------------------------------------------------------------------------------------------
// row_warps warps to a row.  Mean and variance in two passes over the registers: each warp has the mean of its own part and the
// squares around it, and the parts are merged with their counts (exact for any offset of the row, one barrier).
template <typename T, typename TP, int V, int VPT, int MAXT>
__global__ void __launch_bounds__(MAXT) clear_norm_fwd_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float2 s_part[2][32][kMaxRowWarps * 2];
    const RowGroup g(p.row_warps);
    const int first_vec = g.warp * 32 + g.lane, step_vec = p.row_warps * 32;
    int count = 0;  // channels of this warp
#pragma unroll
    for (int v = 0; v < VPT; ++v) count += min(32, max(0, p.n_vec - v * step_vec - g.warp * 32)) * V;
    const float inv_count = count ? 1.f / (float)count : 0.f, inv_c = 1.f / (float)p.C;
    int parity = 0;
    for (unsigned row = blockIdx.x * (unsigned)p.groups + g.grp; row < p.rows; row += gridDim.x * (unsigned)p.groups, parity ^= 1) {
        const unsigned b = row / p.n_rows_b, n = row - b * p.n_rows_b;
        const T *x = static_cast<const T *>(p.x) + (long long)b * p.x_stride_b + (long long)n * p.x_stride_n;
        Pack<T, V> raw[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int i = first_vec + v * step_vec;
            if (i < p.n_vec) raw[v].load(x + (long long)i * V);
            else raw[v].zero();
        }
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float e[V];
            raw[v].get(e);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += e[j];
        }
        float mean = warp_sum(sum) * inv_count, m2 = 0.f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            if (first_vec + v * step_vec < p.n_vec) {
                float e[V];
                raw[v].get(e);
#pragma unroll
                for (int j = 0; j < V; ++j) m2 = fmaf(e[j] - mean, e[j] - mean, m2);
            }
        }
        m2 = warp_sum(m2);
        if (p.row_warps > 1) {
            float2 *part = s_part[parity][g.grp];
            if (g.lane == 0) {
                part[2 * g.warp] = make_float2(mean, m2);
                part[2 * g.warp + 1].x = (float)count;
            }
            group_barrier(1 + g.grp, p.row_warps * 32);
            float2 mine = make_float2(0.f, 0.f);
            float n_mine = 0.f;
            if (g.lane < p.row_warps) {
                mine = part[2 * g.lane];
                n_mine = part[2 * g.lane + 1].x;
            }
            mean = warp_sum(n_mine * mine.x) * inv_c;
            m2 = warp_sum(fmaf(n_mine * (mine.x - mean), mine.x - mean, mine.y));
        }
        const float rstd = rsqrtf(fmaf(m2, inv_c, p.eps));
        if (g.warp == 0 && g.lane == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        const TP *w = static_cast<const TP *>(p.weight), *bias = static_cast<const TP *>(p.bias);
        if (w) w += (long long)b * p.w_stride_b;
        if (bias) bias += (long long)b * p.bias_stride_b;
        T *y = static_cast<T *>(p.out) + (long long)b * p.out_stride_b + (long long)n * p.out_stride_n;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int i = first_vec + v * step_vec;
            if (i < p.n_vec) {
                float e[V];
                raw[v].get(e);
#pragma unroll
                for (int j = 0; j < V; ++j) e[j] = (e[j] - mean) * rstd;
                if (w) {
                    Pack<TP, V> pw;
                    float f[V];
                    pw.load(w + i * V);
                    pw.get(f);
#pragma unroll
                    for (int j = 0; j < V; ++j) e[j] *= p.offset + f[j];
                }
                if (bias) {
                    Pack<TP, V> pb;
                    float f[V];
                    pb.load(bias + i * V);
                    pb.get(f);
#pragma unroll
                    for (int j = 0; j < V; ++j) e[j] += f[j];
                }
                raw[v].set(e);
                raw[v].store(y + (long long)i * V);
            }
        }
    }
}

// Sum over a block of 256 threads, known to all of them.
__device__ __forceinline__ float block_sum(float x, float (&buf)[8])
{
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = x;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += buf[i];
    return t;
}

// Rows too long for registers: a block to a row, read again from the caches for each pass.
template <typename T, typename TP>
__global__ void __launch_bounds__(256) clear_norm_fwd_long_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float buf[8];
    for (unsigned row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const unsigned b = row / p.n_rows_b, n = row - b * p.n_rows_b;
        const T *x = static_cast<const T *>(p.x) + (long long)b * p.x_stride_b + (long long)n * p.x_stride_n;
        T *y = static_cast<T *>(p.out) + (long long)b * p.out_stride_b + (long long)n * p.out_stride_n;
        const TP *w = p.weight ? static_cast<const TP *>(p.weight) + (long long)b * p.w_stride_b : nullptr;
        const TP *bias = p.bias ? static_cast<const TP *>(p.bias) + (long long)b * p.bias_stride_b : nullptr;
        float sum = 0.f, m2 = 0.f;
        for (int i = threadIdx.x; i < p.C; i += 256) sum += (float)x[i];
        const float mean = block_sum(sum, buf) / (float)p.C;
        for (int i = threadIdx.x; i < p.C; i += 256) {
            const float e = (float)x[i] - mean;
            m2 = fmaf(e, e, m2);
        }
        const float rstd = rsqrtf(block_sum(m2, buf) / (float)p.C + p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        for (int i = threadIdx.x; i < p.C; i += 256) {
            float e = ((float)x[i] - mean) * rstd;
            if (w) e *= p.offset + (float)w[i];
            if (bias) e += (float)bias[i];
            y[i] = (T)e;
        }
    }
}

// ---- backward --------------------------------------------------------------------------------------------------------
// A thread keeps its channels for all rows of its group, so the sums of the weights' gradients stay in registers; the groups of
// a block are added in shared memory, the blocks' sums by clear_norm_reduce_kernel in a fixed order.
template <typename T, typename TP, int V, int VPT>
__global__ void __launch_bounds__(512) clear_norm_bwd_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float2 s_part[2][16][kMaxRowWarps];
    extern __shared__ float s_sum[];  // [C] twice: sums of the block's groups
    const RowGroup g(p.row_warps);
    const int first_vec = g.warp * 32 + g.lane, step_vec = p.row_warps * 32;
    const float inv_c = 1.f / (float)p.C;
    const unsigned batch = blockIdx.y;  // 0 where all rows share the weights
    const unsigned rows = p.per_batch ? p.n_rows_b : p.rows;
    float dw[VPT][V], db[VPT][V], gain[VPT][V];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int i = first_vec + v * step_vec;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            dw[v][j] = db[v][j] = 0.f;
            gain[v][j] = 1.f;
        }
        if (p.weight && i < p.n_vec) {
            Pack<TP, V> pw;
            pw.load(static_cast<const TP *>(p.weight) + (long long)batch * p.w_stride_b + i * V);
            pw.get(gain[v]);
#pragma unroll
            for (int j = 0; j < V; ++j) gain[v][j] += p.offset;
        }
    }
    int parity = 0;
    for (unsigned r = blockIdx.x * (unsigned)p.groups + g.grp; r < rows; r += gridDim.x * (unsigned)p.groups, parity ^= 1) {
        const unsigned b = p.per_batch ? batch : r / p.n_rows_b, n = p.per_batch ? r : r - b * p.n_rows_b;
        const T *x = static_cast<const T *>(p.x) + (long long)b * p.x_stride_b + (long long)n * p.x_stride_n;
        const T *dy = static_cast<const T *>(p.dy) + (long long)b * p.dy_stride_b + (long long)n * p.dy_stride_n;
        Pack<T, V> rx[VPT], rd[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int i = first_vec + v * step_vec;
            if (i < p.n_vec) {
                rx[v].load(x + (long long)i * V);
                rd[v].load(dy + (long long)i * V);
            } else {
                rx[v].zero();
                rd[v].zero();
            }
        }
        const size_t stat = (size_t)b * p.n_rows_b + n;
        const float mean = p.mean_in[stat], rstd = p.rstd_in[stat];
        float a = 0.f, c = 0.f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float e[V], d[V];
            rx[v].get(e);
            rd[v].get(d);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float h = (e[j] - mean) * rstd, gr = d[j] * gain[v][j];
                dw[v][j] = fmaf(d[j], h, dw[v][j]);
                db[v][j] += d[j];
                a += gr;
                c = fmaf(gr, h, c);
            }
        }
        a = warp_sum(a);
        c = warp_sum(c);
        if (p.row_warps > 1) {
            float2 *part = s_part[parity][g.grp];
            if (g.lane == 0) part[g.warp] = make_float2(a, c);
            group_barrier(1 + g.grp, p.row_warps * 32);
            const float2 mine = g.lane < p.row_warps ? part[g.lane] : make_float2(0.f, 0.f);
            a = warp_sum(mine.x);
            c = warp_sum(mine.y);
        }
        a *= inv_c;
        c *= inv_c;
        T *dx = static_cast<T *>(p.out) + (long long)b * p.out_stride_b + (long long)n * p.out_stride_n;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int i = first_vec + v * step_vec;
            if (i < p.n_vec) {
                float e[V], d[V];
                rx[v].get(e);
                rd[v].get(d);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float h = (e[j] - mean) * rstd;
                    e[j] = rstd * (fmaf(d[j], gain[v][j], -a) - h * c);
                }
                rx[v].set(e);
                rx[v].store(dx + (long long)i * V);
            }
        }
    }
    if (!p.partial) return;
    float *out = p.partial + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.C;
    for (int turn = 0; turn < p.groups; ++turn) {  // one group after the other: a fixed order of the sums
        if (g.grp == turn) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int i = first_vec + v * step_vec;
                if (i < p.n_vec) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int col = i * V + j;
                        float w = dw[v][j], bb = db[v][j];
                        if (turn > 0) {
                            w += s_sum[col];
                            bb += s_sum[p.C + col];
                        }
                        if (turn == p.groups - 1) {
                            out[col] = w;
                            out[p.C + col] = bb;
                        } else {
                            s_sum[col] = w;
                            s_sum[p.C + col] = bb;
                        }
                    }
                }
            }
        }
        if (turn + 1 < p.groups) __syncthreads();
    }
}

// Rows too long for registers: the rows' gradients first (a block to a row) ...
template <typename T, typename TP>
__global__ void __launch_bounds__(256) clear_norm_bwd_long_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float buf[8];
    for (unsigned row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const unsigned b = row / p.n_rows_b, n = row - b * p.n_rows_b;
        const T *x = static_cast<const T *>(p.x) + (long long)b * p.x_stride_b + (long long)n * p.x_stride_n;
        const T *dy = static_cast<const T *>(p.dy) + (long long)b * p.dy_stride_b + (long long)n * p.dy_stride_n;
        T *dx = static_cast<T *>(p.out) + (long long)b * p.out_stride_b + (long long)n * p.out_stride_n;
        const TP *w = p.weight ? static_cast<const TP *>(p.weight) + (long long)b * p.w_stride_b : nullptr;
        const float mean = p.mean_in[row], rstd = p.rstd_in[row];
        float a = 0.f, c = 0.f;
        for (int i = threadIdx.x; i < p.C; i += 256) {
            const float gr = (float)dy[i] * (w ? p.offset + (float)w[i] : 1.f);
            a += gr;
            c = fmaf(gr, ((float)x[i] - mean) * rstd, c);
        }
        a = block_sum(a, buf) / (float)p.C;
        c = block_sum(c, buf) / (float)p.C;
        for (int i = threadIdx.x; i < p.C; i += 256) {
            const float gr = (float)dy[i] * (w ? p.offset + (float)w[i] : 1.f);
            dx[i] = (T)(rstd * (gr - a - ((float)x[i] - mean) * rstd * c));
        }
    }
}

// ... and before them, as dx may lie in the place of x or dy, the sums of their columns: a thread to a channel, blockIdx.y a share
// of the rows, blockIdx.z the batch entry (0 where all rows share the weights).
template <typename T>
__global__ void __launch_bounds__(256) clear_norm_columns_kernel(const __grid_constant__ NormParams p)
{
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= p.C) return;
    const unsigned rows = p.per_batch ? p.n_rows_b : p.rows;
    float dw = 0.f, db = 0.f;
    for (unsigned r = blockIdx.y; r < rows; r += gridDim.y) {
        const unsigned b = p.per_batch ? blockIdx.z : r / p.n_rows_b, n = p.per_batch ? r : r - b * p.n_rows_b;
        const size_t stat = (size_t)b * p.n_rows_b + n;
        const float x = (float)static_cast<const T *>(p.x)[(long long)b * p.x_stride_b + (long long)n * p.x_stride_n + col];
        const float dy = (float)static_cast<const T *>(p.dy)[(long long)b * p.dy_stride_b + (long long)n * p.dy_stride_n + col];
        dw = fmaf(dy, (x - p.mean_in[stat]) * p.rstd_in[stat], dw);
        db += dy;
    }
    float *out = p.partial + ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * 2 * p.C;
    out[col] = dw;
    out[p.C + col] = db;
}

// Sums of the blocks' partial sums [parts][2][C], 32 channels and 8 shares of the parts to a block, in a fixed order.
template <typename TP>
__global__ void __launch_bounds__(256)
clear_norm_reduce_kernel(const float *partial, int parts, int C, TP *dweight, TP *dbias, long long dw_stride_b, long long db_stride_b)
{
    __shared__ float s[8][33];
    ptx::grid_wait();
    const int lane = threadIdx.x & 31, share = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    TP *out = blockIdx.z == 0 ? dweight : dbias;
    if (!out) return;
    out += (long long)blockIdx.y * (blockIdx.z == 0 ? dw_stride_b : db_stride_b);
    const float *src = partial + ((size_t)blockIdx.y * parts * 2 + blockIdx.z) * C + col;
    float sum = 0.f;
    if (col < C)
        for (int i = share; i < parts; i += 8) sum += src[(size_t)i * 2 * C];
    s[share][lane] = sum;
    __syncthreads();
    if (share == 0 && col < C) {
#pragma unroll
        for (int i = 1; i < 8; ++i) sum += s[i][lane];
        out[col] = (TP)sum;
    }
}

// ---- launches --------------------------------------------------------------------------------------------------------

int sm_count(int *n)
{
    int dev = 0;
    CLEAR_CUDA_TRY(cudaGetDevice(&dev));
    CLEAR_CUDA_TRY(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
    return CLEAR_OK;
}

// Accesses of V channels are possible where every row of every tensor begins on their boundary.
bool vector_fits(const NormArgs &a, int V, size_t elem, size_t param_elem)
{
    if (a.C % V) return false;
    auto strides = [&](long long sb, long long sn) { return (a.B == 1 || sb % V == 0) && (a.N == 1 || sn % V == 0); };
    const size_t bytes = std::min<size_t>(16, V * elem), pbytes = std::min<size_t>(16, V * param_elem);
    if (!aligned_to(a.x, bytes) || !aligned_to(a.out, bytes) || !strides(a.x_stride_b, a.x_stride_n) ||
        !strides(a.out_stride_b, a.out_stride_n))
        return false;
    if (a.dy && (!aligned_to(a.dy, bytes) || !strides(a.dy_stride_b, a.dy_stride_n))) return false;
    if (a.weight && (!aligned_to(a.weight, pbytes) || (a.B > 1 && a.w_stride_b % V))) return false;
    if (a.bias && (!aligned_to(a.bias, pbytes) || (a.B > 1 && a.bias_stride_b % V))) return false;
    return true;
}

NormParams params_of(const NormArgs &a)
{
    NormParams p{};
    p.x = a.x; p.dy = a.dy; p.out = a.out; p.weight = a.weight; p.bias = a.bias;
    p.mean_in = a.mean_in; p.rstd_in = a.rstd_in; p.mean = a.mean; p.rstd = a.rstd;
    p.x_stride_b = a.x_stride_b; p.x_stride_n = a.x_stride_n;
    p.dy_stride_b = a.dy_stride_b; p.dy_stride_n = a.dy_stride_n;
    p.out_stride_b = a.out_stride_b; p.out_stride_n = a.out_stride_n;
    p.w_stride_b = a.w_stride_b; p.bias_stride_b = a.bias_stride_b;
    p.rows = (unsigned)((long long)a.B * a.N);
    p.n_rows_b = (unsigned)a.N;
    p.C = a.C;
    p.per_batch = a.per_batch;
    p.offset = a.offset;
    p.eps = a.eps;
    return p;
}

template <typename T, typename TP, int V, int VPT>
int launch_fwd(NormParams p, int n_sm, cudaStream_t stream)
{
    p.n_vec = p.C / V;
    p.row_warps = (p.n_vec + 32 * VPT - 1) / (32 * VPT);
    p.groups = p.row_warps >= 8 ? 1 : 8 / p.row_warps;
    const int threads = p.groups * p.row_warps * 32;
    const long long need = ((long long)p.rows + p.groups - 1) / p.groups;
    auto go = [&](auto kernel) -> int {
        int per_sm = 0;
        CLEAR_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0));
        kernel<<<(unsigned)std::min<long long>(need, (long long)n_sm * std::max(1, per_sm)), threads, 0, stream>>>(p);
        CLEAR_CUDA_TRY(cudaGetLastError());
        return CLEAR_OK;
    };
    return threads <= 256 ? go(clear_norm_fwd_kernel<T, TP, V, VPT, 256>) : go(clear_norm_fwd_kernel<T, TP, V, VPT, 512>);
}

template <typename T, typename TP>
int norm_fwd(const NormArgs &a, cudaStream_t stream)
{
    constexpr int kWide = 16 / (int)sizeof(T);
    int n_sm = 0;
    if (const int rc = sm_count(&n_sm)) return rc;
    NormParams p = params_of(a);
    if (vector_fits(a, kWide, sizeof(T), sizeof(TP))) {
        const int n_vec = a.C / kWide;
        if (n_vec <= 32 * 1) return launch_fwd<T, TP, kWide, 1>(p, n_sm, stream);
        if (n_vec <= 32 * 2) return launch_fwd<T, TP, kWide, 2>(p, n_sm, stream);
        if (n_vec <= 32 * 4) return launch_fwd<T, TP, kWide, 4>(p, n_sm, stream);
        if (n_vec <= 32 * kMaxRowWarps * 8) return launch_fwd<T, TP, kWide, 8>(p, n_sm, stream);
    } else {
        if (a.C <= 32 * kMaxRowWarps * 4) return launch_fwd<T, TP, 1, 4>(p, n_sm, stream);
        if (a.C <= 32 * kMaxRowWarps * 16) return launch_fwd<T, TP, 1, 16>(p, n_sm, stream);
    }
    clear_norm_fwd_long_kernel<T, TP><<<(unsigned)std::min<long long>(p.rows, 8LL * n_sm), 256, 0, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    return CLEAR_OK;
}

template <typename TP>
int launch_reduce(const NormArgs &a, int parts, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((a.C + 31) / 32, a.per_batch ? a.B : 1, 2);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    CLEAR_CUDA_TRY(cudaLaunchKernelEx(&cfg, clear_norm_reduce_kernel<TP>, (const float *)a.workspace, parts, a.C,
                                      static_cast<TP *>(a.dweight), static_cast<TP *>(a.dbias), a.dw_stride_b, a.db_stride_b));
    return CLEAR_OK;
}

template <typename T, typename TP, int V, int VPT>
int launch_bwd(NormParams p, const NormArgs &a, int parts, cudaStream_t stream)
{
    p.n_vec = p.C / V;
    p.row_warps = (p.n_vec + 32 * VPT - 1) / (32 * VPT);
    p.groups = std::max(1, std::min(15, 16 / p.row_warps));
    const bool sums = a.dweight || a.dbias;
    p.partial = sums ? static_cast<float *>(a.workspace) : nullptr;
    const size_t smem = sums && p.groups > 1 ? 2 * sizeof(float) * (size_t)p.C : 0;
    auto kernel = clear_norm_bwd_kernel<T, TP, V, VPT>;
    if (smem > 40 * 1024)
        CLEAR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    kernel<<<dim3((unsigned)parts, a.per_batch ? a.B : 1), p.groups * p.row_warps * 32, smem, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    return sums ? launch_reduce<TP>(a, parts, stream) : CLEAR_OK;
}

template <typename T, typename TP>
int norm_bwd(const NormArgs &a, int parts, int n_sm, cudaStream_t stream)
{
    constexpr int kWide = 16 / (int)sizeof(T);
    NormParams p = params_of(a);
    if (vector_fits(a, kWide, sizeof(T), sizeof(TP))) {
        const int n_vec = a.C / kWide;
        if (n_vec <= 32 * kMaxRowWarps) return launch_bwd<T, TP, kWide, 1>(p, a, parts, stream);
        if (n_vec <= 32 * kMaxRowWarps * 16 / kWide) return launch_bwd<T, TP, kWide, 16 / kWide>(p, a, parts, stream);
    } else {
        if (a.C <= 32 * kMaxRowWarps * 4) return launch_bwd<T, TP, 1, 4>(p, a, parts, stream);
        if (a.C <= 32 * kMaxRowWarps * 16) return launch_bwd<T, TP, 1, 16>(p, a, parts, stream);
    }
    if (a.dweight || a.dbias) {
        p.partial = static_cast<float *>(a.workspace);
        clear_norm_columns_kernel<T><<<dim3((a.C + 255) / 256, parts, a.per_batch ? a.B : 1), 256, 0, stream>>>(p);
        CLEAR_CUDA_TRY(cudaGetLastError());
        if (const int rc = launch_reduce<TP>(a, parts, stream)) return rc;
    }
    clear_norm_bwd_long_kernel<T, TP><<<(unsigned)std::min<long long>(p.rows, 8LL * n_sm), 256, 0, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    return CLEAR_OK;
}

// Blocks a weight's rows are shared over, a partial sum each: one block an SM over all weights, and no more than rows.
int bwd_parts(int B, int N, int per_batch, int n_sm)
{
    const long long weights = per_batch ? B : 1, rows = per_batch ? N : (long long)B * N;
    return (int)std::max<long long>(1, std::min<long long>(rows, (n_sm + weights - 1) / weights));
}

}  // namespace

int norm_bwd_workspace(int B, int N, int C, int per_batch, size_t *bytes)
{
    int n_sm = 0;
    if (const int rc = sm_count(&n_sm)) return rc;
    *bytes = (size_t)bwd_parts(B, N, per_batch, n_sm) * (per_batch ? B : 1) * 2 * sizeof(float) * (size_t)C;
    return CLEAR_OK;
}

int launch_norm_fwd(const NormArgs &a, cudaStream_t stream)
{
    if (a.dtype == CLEAR_F32) return norm_fwd<float, float>(a, stream);
    return a.param_dtype == CLEAR_F32 ? norm_fwd<__nv_bfloat16, float>(a, stream) : norm_fwd<__nv_bfloat16, __nv_bfloat16>(a, stream);
}

int launch_norm_bwd(const NormArgs &a, cudaStream_t stream)
{
    int n_sm = 0;
    if (const int rc = sm_count(&n_sm)) return rc;
    const int parts = bwd_parts(a.B, a.N, a.per_batch, n_sm);
    if (a.dtype == CLEAR_F32) return norm_bwd<float, float>(a, parts, n_sm, stream);
    return a.param_dtype == CLEAR_F32 ? norm_bwd<__nv_bfloat16, float>(a, parts, n_sm, stream)
                                      : norm_bwd<__nv_bfloat16, __nv_bfloat16>(a, parts, n_sm, stream);
}

}  // namespace clear
