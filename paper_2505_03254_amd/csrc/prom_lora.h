// The ternary pointwise layer with low-rank adapters of many requests: what its kernel files share.
//
// Forward, l the adapter of a row's batch element:
//   hid = step * (x a_l^T) [rows][rank],  y = (acc * w_scale) * step + bias + scale_l * (hid b_l)
// Backward:
//   g = scale_l * (dy b_l^T),  dx = (dy * w_scale) W + g a_l,  da_l = sum (g * step) x,  db_l = scale_l * sum hid dy
//
// The adapters' products run on the bf16 matrix cores whatever the types: a real factor is split into bf16 planes
// (v = v0 + v1 + v2, each the rounding of what is left: 8, 16, 24 bits), products of planes are exact in float32, and as many planes are
// taken as the result's type can tell apart.  int8 activations are exact in one plane, bf16 in one, f16 in two.
//
// dy * w_scale is no bf16 number even where dy is, so for a bf16 dy one plane of bf16 would lose as much as the rounding of dx itself (norm of the
// error 1.2 to 1.4 times that of one rounding).  Its plane is f16 instead, 11 bits at the same rate, and a power of two per row brings the row's
// largest product to [2^14, 2^15): f16's exponents hold the 28 binades below that with all bits and 10 more with fewer.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "prom.h"
#include "prom_float.h"

namespace prom {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef int v4i_u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kLoraMaxRank = 128;
constexpr int kLoraMaxChannels = 65536;  // |64 * acc| < 2^31 and |acc| < 2^24 exact in float32
constexpr int kLoraMaxAdapters = 65535;
constexpr long long kLoraMaxRows = 1LL << 26;  // a launch has fewer than 2^32 threads: 512 for 16 rows

// Planes of a type; of the products of two split numbers those are taken that reach 2^-24 of the whole.
template <typename T> constexpr int planes_of() { return sizeof(T) == 4 ? 3 : std::is_same<T, bf16_t>::value ? 1 : 2; }

template <int P> __device__ __forceinline__ void split(float v, bf16_t (&out)[P])
{
#pragma unroll
    for (int p = 0; p < P; ++p) {
        out[p] = (bf16_t)v;
        if (p + 1 < P) v -= (float)out[p];
    }
    // an infinity or a NaN stands in the first plane alone (inf - inf would put a NaN beside it)
    if constexpr (P > 1) {
        const float first = (float)out[0];
        if (!(fabsf(first) <= 0x1.fffffep127f)) {
#pragma unroll
            for (int p = 1; p < P; ++p) out[p] = (bf16_t)0.0f;
        }
    }
}
template <int P, typename T, int N> __device__ __forceinline__ void split_piece(const Piece<T, N> &v, v8bf (&out)[P])
{
    static_assert(N == 8, "a fragment");
    if constexpr (P == 1 && std::is_same<T, bf16_t>::value) {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[0][e] = v.e[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16_t s[P];
            split<P>((float)v.e[e], s);
#pragma unroll
            for (int p = 0; p < P; ++p) out[p][e] = s[p];
        }
    }
}

__device__ __forceinline__ v4f mfma_bf16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f mfma_f16(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The type of dy whose planes are one f16 with a factor per row.
template <typename T> constexpr bool kScaledPlane = std::is_same<T, bf16_t>::value;
// Factor of a row whose largest |dy * w_scale| is `most` (a NaN's bits above all), and its inverse halved: the codes stand for twice their
// values.  Both are powers of two within float32's normal range; an infinity or a NaN stays what it is.
__device__ __forceinline__ float plane_up(float most)
{
    const int e = __float_as_int(most) >> 23;  // biased exponent, no sign
    return __int_as_float((min(141 - e, 125) + 127) << 23);
}
__device__ __forceinline__ float plane_down(float up) { return __int_as_float((253 << 23) - __float_as_int(up)); }  // 0.5 / up

// Rows sorted by adapter: where each one's begin, and tiles of them that hold one adapter only.  Row positions are
// counted in sorted order; elements without an adapter come last as group `adapters`.
struct LoraPlan {
    int *order;    // [n] batch elements in sorted order
    int *rows;     // [m] row numbers in sorted order
    int2 *groups;  // [adapters + 1] first position, rows
    int4 *tiles;   // [m / tile + adapters + 1] group, first position, rows, 0
    int4 *chunks;  // [m / chunk + adapters + 1] the same in tiles of `chunk` rows, or NULL
    int tile, chunk;
};

struct LoraGemmArgs {
    const void *x;       // int8 [m][K], or planes [m][planes][Kp]: bf16, or f16 scaled row by row
    const uint32_t *wq;  // packed [Nc][KW]
    const int *rows;     // row numbers by position (not looked at for a few rows)
    const int *index;    // adapter by batch element
    const float *step, *w_scale, *bias;  // (int8 input)
    const float *down;   // [m] what a scaled row's sums are multiplied by
    const float *hid;    // [m][rank] scaled by the adapter's scale here (scale != NULL) or already
    const float *scale;
    const void *low;     // [adapters][rank][Nc]
    const void *first;   // [adapters][rank][K] (a few rows that form hid themselves)
    float *hid_out;
    void *y;
    int m, hw, K, KW, Nc, rank, adapters, planes, Kp;
};

}  // namespace prom
