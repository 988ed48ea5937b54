// Device helpers of the kernels that take real-valued tensors: element types, 16-byte pieces, wavefront sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "prom.h"

namespace prom {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

// Element types behind PROM_F32, PROM_BF16 and PROM_F16.
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline int type_bytes(int type) { return type == PROM_F32 ? 4 : type == PROM_BF16 || type == PROM_F16 ? 2 : 0; }

// A pointer known to point to global memory.  One that comes out of memory may point anywhere to the compiler, and its flat accesses
// wait for LDS as well as for each other (AdamW, whose pointers stand in a table, 75 M elements in 8 bits: 257 us flat, 252 global).
template <typename T> using Global = T __attribute__((address_space(1)));

// A piece of 16 (8, 4) bytes at an address that is aligned to its elements only: gfx950 loads and stores dwords at any
// byte address, and the row of an odd width starts anywhere.
template <typename T, int N> struct Piece {
    typedef T Vec __attribute__((ext_vector_type(N)));
    typedef Vec Loose __attribute__((aligned(sizeof(T))));
    struct __attribute__((packed, aligned(sizeof(T)))) Raw { T e[N]; };
    T e[N];
    __device__ __forceinline__ void load(const T *p)
    {
        const Raw r = *reinterpret_cast<const Raw *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = r.e[i];
    }
    __device__ __forceinline__ void load(const Global<T> *p)
    {
        const Vec v = *reinterpret_cast<const Global<Loose> *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = v[i];
    }
    __device__ __forceinline__ void store(T *p) const
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < N; ++i) r.e[i] = e[i];
        *reinterpret_cast<Raw *>(p) = r;
    }
    __device__ __forceinline__ void store(Global<T> *p) const
    {
        Vec v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = e[i];
        *reinterpret_cast<Global<Loose> *>(p) = v;
    }
    // the first `have` elements (have may be anything); the others read as zero and are not written
    template <typename P> __device__ __forceinline__ void load_some(P p, int have)
    {
        if (have >= N) load(p);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                e[i] = (T)0.0f;
                if (i < have) e[i] = p[i];
            }
        }
    }
    // The same by loads without a test each, the first element in the place of absent ones: they are in flight together, where those
    // of load_some wait for one another (the halves of a register).  It holds N more registers, so only kernels that have them call it:
    // the adapters' gradients (5341 rows of 513 channels in bf16 24 -> 14 us); the large products spill with it.
    template <typename P> __device__ __forceinline__ void load_some_at_once(P p, int have)
    {
        if constexpr (sizeof(T) == 4) load_some(p, have);  // (a register each: nothing waits there)
        else if (have >= N) load(p);
        else if (have > 0) {
            T v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = p[i < have ? i : 0];
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = i < have ? v[i] : (T)0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = (T)0.0f;
        }
    }
    template <typename P> __device__ __forceinline__ void store_some(P p, int have) const
    {
        if (have >= N) store(p);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < have) p[i] = e[i];
        }
    }
};

// Float32 operations that are rounded one by one whatever stands around them (the compiler contracts a product and the sum
// behind it into one operation otherwise, the header's __fmul_rn and __fadd_rn included).
__device__ __forceinline__ float mul_f32(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ float add_f32(float a, float b)
{
#pragma clang fp contract(off)
    return a + b;
}
__device__ __forceinline__ float sub_f32(float a, float b)
{
#pragma clang fp contract(off)
    return a - b;
}

// correctly rounded (the header's __fsqrt_rn is not)
__device__ __forceinline__ float sqrt_f32(float a) { return __builtin_sqrtf(a); }

// The same for 0, 2^-96 and above, infinities and NaN.  The instruction's result s is off by one step at most; with d and u
// its neighbours, the root lies below the middle of d and s where d * s >= a (the middle's square is d * s and a quarter of
// a step's square more), above that of s and u where s * u < a.  sqrt_f32 scales small arguments as well: 14 instructions against 9.
__device__ __forceinline__ float sqrt_large_f32(float a)
{
    const float s = __builtin_amdgcn_sqrtf(a);
    const float d = __int_as_float(__float_as_int(s) - 1), u = __int_as_float(__float_as_int(s) + 1);
    const float below = __builtin_fmaf(-d, s, a), above = __builtin_fmaf(-u, s, a);
    float r = below <= 0.0f ? d : s;
    return above > 0.0f ? u : r;
}

// Sum and maximum over the 64 lanes, the same in every lane and the same from run to run.  Five steps inside rows
// and between them by DPP, whose latency is that of an addition (a shuffle through LDS takes 64 cycles and more).
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_f32(float v, float fill)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(fill), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <typename Op> __device__ __forceinline__ float wave_reduce(float v, float none, Op op)
{
    v = op(v, dpp_f32<0x111, 0xf>(v, none));  // row_shr:1
    v = op(v, dpp_f32<0x112, 0xf>(v, none));  // row_shr:2
    v = op(v, dpp_f32<0x114, 0xf>(v, none));  // row_shr:4
    v = op(v, dpp_f32<0x118, 0xf>(v, none));  // row_shr:8
    v = op(v, dpp_f32<0x142, 0xa>(v, none));  // row_bcast:15 into rows 1 and 3
    v = op(v, dpp_f32<0x143, 0xc>(v, none));  // row_bcast:31 into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_sum_f32(float v)
{
    return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
// maximum of non-negative values or NaN by their bits, in which a NaN is larger than everything
__device__ __forceinline__ float bits_max(float a, float b)
{
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}
__device__ __forceinline__ float wave_max_bits(float v)
{
    return wave_reduce(v, 0.0f, [](float a, float b) { return bits_max(a, b); });
}
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_f64(double v)
{
    const long long b = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}
__device__ __forceinline__ double wave_sum_f64(double v)
{
    v += dpp_f64<0x111, 0xf>(v);
    v += dpp_f64<0x112, 0xf>(v);
    v += dpp_f64<0x114, 0xf>(v);
    v += dpp_f64<0x118, 0xf>(v);
    v += dpp_f64<0x142, 0xa>(v);
    v += dpp_f64<0x143, 0xc>(v);
    const long long b = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_readlane((int)b, 63);
    const int hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}

// Workgroup barrier that orders LDS traffic only: loads of global memory stay on their way across it.
__device__ __forceinline__ void lds_only_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- host ------------------------------------------------------------------------------------
inline bool misaligned(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) != 0; }

struct Range {
    const void *p;  // NULL: none
    size_t n;
};
inline bool ranges_meet(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
}
// Whether an output shares a byte with an input or with another output.
inline bool outputs_meet(const Range *out, int outs, const Range *in, int ins)
{
    for (int i = 0; i < outs; ++i) {
        for (int k = 0; k < ins; ++k)
            if (ranges_meet(out[i], in[k])) return true;
        for (int k = 0; k < i; ++k)
            if (ranges_meet(out[i], out[k])) return true;
    }
    return false;
}

}  // namespace prom
