// Rotary positions of Q and K: each pair of channels turns by position * frequency, over all or the first part of a head; the
// gradient is the turn by the opposite angle.  Pairs are neighbours (2p, 2p+1) or half the rotary part apart (p, p + P).
//
// HBM bounds it (every element in once, out once).  A thread owns a few pairs of one token and walks over the heads: angles
// depend on the token only, so their sines and cosines are computed once and serve all heads of Q and of K.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "clear_internal.hpp"
#include "rope_angle.cuh"
#include "row_io.cuh"

namespace clear {
namespace {

constexpr int kRopeThreads = 256;

struct RopeTensor {
    const void *in;
    void *out;
    long long in_b, in_h, in_n, out_b, out_h, out_n;
    int heads;
    int copy;  // whether the channels behind the rotary part have to be copied
};

struct RopeParams {
    RopeTensor t[2];
    const void *positions;
    long long pos_b, pos_n;
    long long n_items;          // tokens of all batch entries times threads a token
    unsigned n_tokens;          // tokens of a batch entry
    int pos64;
    int pairs, turn_items, items;  // pairs of a head; threads a token: turning, all
    int heads_a_part;           // heads (of Q and K together) that a thread walks over
    int head_dim;
    float factor, sign;
    uint64_t turns[kMaxRopePairs];
    uint8_t axis[kMaxRopePairs];
};

// V channels to an access.  HALF: a thread turns V pairs, two accesses; otherwise max(V, 2) neighbouring channels.
template <typename T, int V, bool HALF>
struct Turn {
    static constexpr int kPairs = HALF ? V : (V > 1 ? V / 2 : 1);
    static constexpr int kAccesses = HALF || V == 1 ? 2 : 1;
    float s[kPairs], c[kPairs];

    static __device__ __forceinline__ int second(int first, int pairs) { return HALF ? first + pairs : first + 1; }

    __device__ __forceinline__ void load(const T *row, int first, int pairs, Pack<T, V> (&x)[kAccesses]) const
    {
        x[0].load(row + first);
        if constexpr (kAccesses == 2) x[1].load(row + second(first, pairs));
    }
    __device__ __forceinline__ void turn_store(T *row, int first, int pairs, Pack<T, V> (&x)[kAccesses]) const
    {
        if constexpr (kAccesses == 2) {
            float a[V], b[V];
            x[0].get(a);
            x[1].get(b);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float lo = a[i] * c[i] - b[i] * s[i], hi = a[i] * s[i] + b[i] * c[i];
                a[i] = lo;
                b[i] = hi;
            }
            x[0].set(a);
            x[1].set(b);
            x[0].store(row + first);
            x[1].store(row + second(first, pairs));
        } else {
            float a[V];
            x[0].get(a);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float lo = a[2 * i] * c[i] - a[2 * i + 1] * s[i], hi = a[2 * i] * s[i] + a[2 * i + 1] * c[i];
                a[2 * i] = lo;
                a[2 * i + 1] = hi;
            }
            x[0].set(a);
            x[0].store(row + first);
        }
    }
};

template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) clear_rope_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int kRows = 4;  // heads in flight
    using Turner = Turn<T, V, HALF>;
    const long long item = (long long)blockIdx.x * kRopeThreads + threadIdx.x;
    if (item >= p.n_items) return;
    const long long token = item / p.items;
    const int part = (int)(item - token * p.items);
    const unsigned b = (unsigned)(token / p.n_tokens), n = (unsigned)(token - (long long)b * p.n_tokens);
    int h0 = blockIdx.y * p.heads_a_part, h1 = h0 + p.heads_a_part;  // of the heads of Q, then those of K
    const bool turning = part < p.turn_items;
    Turner turner;
    int first;
    if (turning) {
        const int pair0 = part * Turner::kPairs;
        first = HALF ? pair0 : 2 * pair0;
        const long long at = (long long)b * p.pos_b + (long long)n * p.pos_n;
#pragma unroll
        for (int i = 0; i < Turner::kPairs; ++i) {
            const int axis = p.axis[pair0 + i];
            const int64_t pos = p.pos64 ? static_cast<const int64_t *>(p.positions)[at + axis]
                                        : (int64_t)static_cast<const int32_t *>(p.positions)[at + axis];
            turn_sincos(pos, p.turns[pair0 + i], turner.s[i], turner.c[i]);
            turner.s[i] *= p.factor * p.sign;
            turner.c[i] *= p.factor;
        }
    } else {
        first = 2 * p.pairs + (part - p.turn_items) * V;
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const RopeTensor &t = p.t[which];
        const int from = max(h0, 0), to = min(h1, t.heads);
        h0 -= t.heads;
        h1 -= t.heads;
        if (from >= to || !(turning || t.copy)) continue;
        const T *in = static_cast<const T *>(t.in) + (long long)b * t.in_b + (long long)n * t.in_n + from * t.in_h;
        T *out = static_cast<T *>(t.out) + (long long)b * t.out_b + (long long)n * t.out_n + from * t.out_h;
        int h = from;
        if (turning) {
            for (; h + kRows <= to; h += kRows) {
                Pack<T, V> x[kRows][Turner::kAccesses];
#pragma unroll
                for (int j = 0; j < kRows; ++j) turner.load(in + j * t.in_h, first, p.pairs, x[j]);
#pragma unroll
                for (int j = 0; j < kRows; ++j) turner.turn_store(out + j * t.out_h, first, p.pairs, x[j]);
                in += kRows * t.in_h;
                out += kRows * t.out_h;
            }
            for (; h < to; ++h) {
                Pack<T, V> x[Turner::kAccesses];
                turner.load(in, first, p.pairs, x);
                turner.turn_store(out, first, p.pairs, x);
                in += t.in_h;
                out += t.out_h;
            }
        } else {
            for (; h + kRows <= to; h += kRows) {
                Pack<T, V> x[kRows];
#pragma unroll
                for (int j = 0; j < kRows; ++j) x[j].load(in + j * t.in_h + first);
#pragma unroll
                for (int j = 0; j < kRows; ++j) x[j].store(out + j * t.out_h + first);
                in += kRows * t.in_h;
                out += kRows * t.out_h;
            }
            for (; h < to; ++h) {
                Pack<T, V> x;
                x.load(in + first);
                x.store(out + first);
                in += t.in_h;
                out += t.out_h;
            }
        }
    }
}

template <typename T, int V, bool HALF>
int launch(RopeParams &p, const RopeArgs &a, int n_sm, cudaStream_t stream)
{
    p.turn_items = p.pairs / Turn<T, V, HALF>::kPairs;
    p.items = p.turn_items + (p.t[0].copy || p.t[1].copy ? (p.head_dim - 2 * p.pairs) / V : 0);
    p.n_items = (long long)a.B * a.N * p.items;
    const long long blocks = (p.n_items + kRopeThreads - 1) / kRopeThreads;
    if (blocks > 0x7fffffffLL) return CLEAR_ERR_UNSUPPORTED;
    // heads are shared out over blocks only while tokens alone leave SMs without work: every share computes the angles anew
    const int heads = p.t[0].heads + p.t[1].heads;
    const int parts = (int)std::min<long long>(heads, std::max<long long>(1, 4LL * n_sm / blocks));
    p.heads_a_part = (heads + parts - 1) / parts;
    const unsigned shares = (unsigned)((heads + p.heads_a_part - 1) / p.heads_a_part);
    clear_rope_kernel<T, V, HALF><<<dim3((unsigned)blocks, shares), kRopeThreads, 0, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    return CLEAR_OK;
}

// Accesses of V channels: rows on their boundary, and the rotary part (its halves) and the head whole numbers of them.
bool fits(const RopeParams &p, int V, size_t elem, bool half)
{
    if ((half ? p.pairs : 2 * p.pairs) % V || p.head_dim % V) return false;
    for (const RopeTensor &t : p.t) {
        if (!t.heads) continue;
        if (!aligned_to(t.in, V * elem) || !aligned_to(t.out, V * elem)) return false;
        for (long long s : {t.in_b, t.in_h, t.in_n, t.out_b, t.out_h, t.out_n})
            if (s % V) return false;
    }
    return true;
}

template <typename T, bool HALF>
int launch_for(RopeParams &p, const RopeArgs &a, int n_sm, cudaStream_t stream)
{
    if (sizeof(T) == 2 && fits(p, 8, sizeof(T), HALF)) return launch<T, sizeof(T) == 2 ? 8 : 4, HALF>(p, a, n_sm, stream);
    if (fits(p, 4, sizeof(T), HALF)) return launch<T, 4, HALF>(p, a, n_sm, stream);
    if (fits(p, 2, sizeof(T), HALF)) return launch<T, 2, HALF>(p, a, n_sm, stream);
    return launch<T, 1, HALF>(p, a, n_sm, stream);
}

}  // namespace

int launch_rope(const RopeArgs &a, cudaStream_t stream)
{
    int dev = 0, n_sm = 0;
    CLEAR_CUDA_TRY(cudaGetDevice(&dev));
    CLEAR_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
    RopeParams p{};
    int pair = 0;
    for (int x = 0; x < a.n_axes; ++x)
        for (int k = 0; k < a.axes_dim[x] / 2; ++k, ++pair) {
            p.turns[pair] = turns_of(a.frequencies[pair]);
            p.axis[pair] = (uint8_t)x;
        }
    p.pairs = pair;
    for (int i = 0; i < 2; ++i) {
        const RopeIo &io = a.io[i];
        RopeTensor &t = p.t[i];
        t.heads = io.in ? io.heads : 0;
        if (!t.heads) continue;
        t.in = io.in;
        t.out = io.out;
        // a stride that no index reaches counts as zero
        auto s = [](long long stride, int n) { return n > 1 ? stride : 0LL; };
        t.in_b = s(io.in_stride_b, a.B); t.in_h = s(io.in_stride_h, io.heads); t.in_n = s(io.in_stride_n, a.N);
        t.out_b = s(io.out_stride_b, a.B); t.out_h = s(io.out_stride_h, io.heads); t.out_n = s(io.out_stride_n, a.N);
        t.copy = io.in != io.out && 2 * pair < a.head_dim;
    }
    p.positions = a.positions;
    p.pos_b = a.pos_stride_b;
    p.pos_n = a.pos_stride_n;
    p.pos64 = a.pos64;
    p.n_tokens = (unsigned)a.N;
    p.head_dim = a.head_dim;
    p.factor = a.factor;
    p.sign = a.inverse ? -1.f : 1.f;
    if (a.dtype == CLEAR_BF16)
        return a.half ? launch_for<__nv_bfloat16, true>(p, a, n_sm, stream) : launch_for<__nv_bfloat16, false>(p, a, n_sm, stream);
    return a.half ? launch_for<float, true>(p, a, n_sm, stream) : launch_for<float, false>(p, a, n_sm, stream);
}

}  // namespace clear
