// Rotary positions of Q and K: each pair of channels turns by position * frequency, over all or the first part of a head; the
// gradient is the turn by the opposite angle.  Pairs are neighbours (2p, 2p+1) or half the rotary part apart (p, p + P).
//
// HBM bounds it (every element in once, out once).  A thread owns a few pairs of one token and walks over heads: angles depend on
// the token only, so their sines and cosines are computed once and serve several heads of Q and of K.  Device time, and bytes over
// the measured copy rate of 6541 GB/s: 66048 tokens of 24 + 8 heads of 128, half of each turned, 169 us, 0.98; packed projection of
// 4608 tokens of 24 + 24 heads 21.4 us, 0.81; fp32 gradient of 16680 tokens of 24 heads of 80 43 us, 0.91; two tokens 2.7 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "clear_internal.hpp"
#include "launch_once.hpp"
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
    long long n_tokens_all;     // tokens of all batch entries
    unsigned n_tokens;          // tokens of a batch entry
    unsigned turn_blocks;       // blocks that turn; those behind them copy
    int narrow;                 // whether tokens times threads fit 32 bits
    int copy_v;                 // channels an access of those
    int pairs, turn_items, copy_items;  // pairs of a head; threads a token
    int heads_a_part;           // heads (of Q and K together) that a thread walks over
    int head_dim;
    float factor, sin_factor;
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

// V channels of each of a token's heads, four heads at a time.
template <typename T, int V>
__device__ __forceinline__ void copy_heads(const T *in, T *out, long long in_h, long long out_h, int heads)
{
    for (int h = 0; h < heads; h += 4) {
        Pack<T, V> x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (h + j < heads) x[j].load(in + j * in_h);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (h + j < heads) x[j].store(out + j * out_h);
        in += 4 * in_h;
        out += 4 * out_h;
    }
}

template <typename T, int V, bool HALF, typename Int>
__global__ void __launch_bounds__(kRopeThreads, 4) clear_rope_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int kRows = HALF ? 2 : 4;  // heads in flight: four accesses of a thread
    using Turner = Turn<T, V, HALF>;
    // from the parameters, lanes that read at places of their own would be served one after the other (4608 tokens: 24 us, so 21.4)
    __shared__ uint64_t s_turns[kMaxRopePairs];
    __shared__ uint8_t s_axis[kMaxRopePairs];
    for (int i = threadIdx.x; i < p.pairs; i += kRopeThreads) {
        s_turns[i] = p.turns[i];
        s_axis[i] = p.axis[i];
    }
    __syncthreads();
    // the first blocks turn, the others copy what does not turn: both kinds of work in one warp would wait for one another
    const bool turning = blockIdx.x < p.turn_blocks;
    const int items = turning ? p.turn_items : p.copy_items;  // threads a token
    const long long item = (long long)(turning ? blockIdx.x : blockIdx.x - p.turn_blocks) * kRopeThreads + threadIdx.x;
    if (item >= p.n_tokens_all * items) return;
    unsigned b, n;
    int part;
    if (p.narrow) {  // 64-bit divisions take their time
        const unsigned token = (unsigned)item / (unsigned)items;
        part = (int)((unsigned)item - token * items);
        b = token / p.n_tokens;
        n = token - b * p.n_tokens;
    } else {
        const long long token = item / items;
        part = (int)(item - token * items);
        b = (unsigned)(token / p.n_tokens);
        n = (unsigned)(token - (long long)b * p.n_tokens);
    }
    int h0 = blockIdx.y * p.heads_a_part, h1 = h0 + p.heads_a_part;  // of the heads of Q, then those of K
    Turner turner;
    int first;
    if (turning) {
        const int pair0 = part * Turner::kPairs;
        first = HALF ? pair0 : 2 * pair0;
        const long long at = (long long)b * p.pos_b + (long long)n * p.pos_n;
        int axis = -1;
        Int pos = 0;
#pragma unroll
        for (int i = 0; i < Turner::kPairs; ++i) {
            if (s_axis[pair0 + i] != axis) {
                axis = s_axis[pair0 + i];
                pos = static_cast<const Int *>(p.positions)[at + axis];
            }
            turn_sincos(pos, s_turns[pair0 + i], turner.s[i], turner.c[i]);
            turner.s[i] *= p.sin_factor;
            turner.c[i] *= p.factor;
        }
    } else {
        first = 2 * p.pairs + part * p.copy_v;
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
        if (!turning) {
            in += first;
            out += first;
            if (p.copy_v * sizeof(T) == 16) copy_heads<T, 16 / sizeof(T)>(in, out, t.in_h, t.out_h, to - from);
            else if (p.copy_v == 4) copy_heads<T, 4>(in, out, t.in_h, t.out_h, to - from);
            else if (p.copy_v == 2) copy_heads<T, 2>(in, out, t.in_h, t.out_h, to - from);
            else copy_heads<T, 1>(in, out, t.in_h, t.out_h, to - from);
            continue;
        }
        int h = from;
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
    }
}

// Accesses of V channels: rows and heads on their boundary, and the part of the head that begins at `offset`.
bool fits(const RopeParams &p, int V, size_t elem, int offset)
{
    if (offset % V || p.head_dim % V) return false;
    for (const RopeTensor &t : p.t) {
        if (!t.heads) continue;
        if (!aligned_to(t.in, V * elem) || !aligned_to(t.out, V * elem)) return false;
        for (long long s : {t.in_b, t.in_h, t.in_n, t.out_b, t.out_h, t.out_n})
            if (s % V) return false;
    }
    return true;
}

template <typename T, int V, bool HALF>
int launch(RopeParams &p, const RopeArgs &a, int n_sm, cudaStream_t stream)
{
    p.turn_items = p.pairs / Turn<T, V, HALF>::kPairs;
    p.copy_v = 16 / (int)sizeof(T);
    while (p.copy_v > 1 && !fits(p, p.copy_v, sizeof(T), 2 * p.pairs)) p.copy_v /= 2;
    p.copy_items = p.t[0].copy || p.t[1].copy ? (p.head_dim - 2 * p.pairs) / p.copy_v : 0;
    p.n_tokens_all = (long long)a.B * a.N;
    p.narrow = p.n_tokens_all * std::max(p.turn_items, p.copy_items) <= 0xffffffffLL - kRopeThreads;
    const long long turn_blocks = (p.n_tokens_all * p.turn_items + kRopeThreads - 1) / kRopeThreads;
    const long long blocks = turn_blocks + (p.n_tokens_all * p.copy_items + kRopeThreads - 1) / kRopeThreads;
    if (blocks > 0x7fffffffLL) return CLEAR_ERR_UNSUPPORTED;
    p.turn_blocks = (unsigned)turn_blocks;
    // Every share of the heads computes the angles anew, which eight heads carry (4608 tokens of 48 heads 21.5 us, all heads in one
    // share 21.8, four 23.1; 16680 of 24 fp32 heads 43.6, 58.8, 42.9); fewer to a share while SMs would be without work.
    const int heads = p.t[0].heads + p.t[1].heads;
    const int parts = (int)std::min<long long>(heads, std::max<long long>((heads + 7) / 8, 4LL * n_sm / blocks));
    p.heads_a_part = std::max((heads + parts - 1) / parts, (heads + 65534) / 65535);
    const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_a_part - 1) / p.heads_a_part));
    if (a.pos64) clear_rope_kernel<T, V, HALF, int64_t><<<grid, kRopeThreads, 0, stream>>>(p);
    else clear_rope_kernel<T, V, HALF, int32_t><<<grid, kRopeThreads, 0, stream>>>(p);
    CLEAR_CUDA_TRY(cudaGetLastError());
    return CLEAR_OK;
}

template <typename T, bool HALF>
int launch_for(RopeParams &p, const RopeArgs &a, int n_sm, cudaStream_t stream)
{
    const int part = HALF ? p.pairs : 2 * p.pairs;  // where the second half of the pairs begins, or the rest of the head
    if (sizeof(T) == 2 && fits(p, 8, sizeof(T), part)) return launch<T, sizeof(T) == 2 ? 8 : 4, HALF>(p, a, n_sm, stream);
    if (fits(p, 4, sizeof(T), part)) return launch<T, 4, HALF>(p, a, n_sm, stream);
    if (fits(p, 2, sizeof(T), part)) return launch<T, 2, HALF>(p, a, n_sm, stream);
    return launch<T, 1, HALF>(p, a, n_sm, stream);
}

}  // namespace

int launch_rope(const RopeArgs &a, cudaStream_t stream)
{
    int device = 0, n_sm = 0;
    if (const int rc = current_sms(&device, &n_sm)) return rc;
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
    p.n_tokens = (unsigned)a.N;
    p.head_dim = a.head_dim;
    p.factor = a.factor;
    p.sin_factor = a.inverse ? -a.factor : a.factor;
    if (a.dtype == CLEAR_BF16)
        return a.half ? launch_for<__nv_bfloat16, true>(p, a, n_sm, stream) : launch_for<__nv_bfloat16, false>(p, a, n_sm, stream);
    return a.half ? launch_for<float, true>(p, a, n_sm, stream) : launch_for<float, false>(p, a, n_sm, stream);
}

}  // namespace clear
