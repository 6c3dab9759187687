// Accesses of V consecutive elements of a row, and reductions, shared by the row-wise kernels (layer norm, rotary positions, the
// gradient of the Q/K preparation).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace clear {

// Two fp32 values in one 64-bit register pair: the packed instructions do both in one issue slot, which is what rows of bf16 at
// HBM speed are short of.
struct F2 {
    unsigned long long v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    explicit __device__ __forceinline__ F2(float both) : F2(both, both) {}
    __device__ __forceinline__ float lo() const { return __uint_as_float((uint32_t)v); }
    __device__ __forceinline__ float hi() const { return __uint_as_float((uint32_t)(v >> 32)); }
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// The same as two registers that need not be neighbours, for values that come one by one.
struct S2 {
    float x, y;
    __device__ __forceinline__ S2() {}
    __device__ __forceinline__ S2(float lo, float hi) : x(lo), y(hi) {}
    explicit __device__ __forceinline__ S2(float both) : x(both), y(both) {}
    __device__ __forceinline__ float lo() const { return x; }
    __device__ __forceinline__ float hi() const { return y; }
};
__device__ __forceinline__ S2 operator+(S2 a, S2 b) { return S2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ S2 operator*(S2 a, S2 b) { return S2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ S2 fma2(S2 a, S2 b, S2 c) { return S2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }

template <int BYTES> struct RawOf;
template <> struct RawOf<2> { using type = unsigned short; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };

// V elements of T as they lie in memory: one access up to 16 bytes, two beyond.
template <typename T, int V>
struct Pack {
    static constexpr int kBytes = (int)sizeof(T) * V;
    static constexpr int kParts = kBytes > 16 ? kBytes / 16 : 1;
    using Raw = typename RawOf<kBytes / kParts>::type;
    Raw raw[kParts];

    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < kParts; ++i) raw[i] = reinterpret_cast<const Raw *>(p)[i];
    }
    __device__ __forceinline__ void store(T *p) const
    {
#pragma unroll
        for (int i = 0; i < kParts; ++i) reinterpret_cast<Raw *>(p)[i] = raw[i];
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kParts; ++i) raw[i] = Raw{};
    }
    __device__ __forceinline__ void get(float (&x)[V]) const
    {
        if constexpr (sizeof(T) == 4) {
            const float *f = reinterpret_cast<const float *>(raw);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = f[i];
        } else if constexpr (V == 1) {
            x[0] = __uint_as_float((uint32_t)raw[0] << 16);   // a bf16 is the upper half of an fp32
        } else {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(raw);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // bf16: rounded once, to nearest even
    __device__ __forceinline__ void set(const float (&x)[V])
    {
        if constexpr (sizeof(T) == 4) {
            float *f = reinterpret_cast<float *>(raw);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = x[i];
        } else if constexpr (V == 1) {
            raw[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
        } else {
            uint32_t *w = reinterpret_cast<uint32_t *>(raw);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
};

// Asynchronous copy of 16 bytes into shared memory where `there` holds, without a branch.
__device__ __forceinline__ void copy_async_if(uint32_t dst, const void *src, bool there)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src),
                 "r"((uint32_t)there)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most LEFT of the thread's latest groups are on their way.
template <int LEFT>
__device__ __forceinline__ void copies_wait()
{
    if constexpr (LEFT == 0) asm volatile("cp.async.wait_all;" ::: "memory");
    else asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Barrier of the `threads` threads of one group of warps (ids 1..15; 0 is __syncthreads).
__device__ __forceinline__ void group_barrier(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

inline bool aligned_to(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; }

}  // namespace clear
