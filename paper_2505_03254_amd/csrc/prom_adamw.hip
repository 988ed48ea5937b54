// One AdamW step over many tensors with one launch, moments in 32 or in 8 bits.
//
//   g = grad * grad_scale,  m' = beta1 m + (1 - beta1) g,  v' = beta2 v + (1 - beta2) g^2
//   p' = p (1 - lr wd) - (lr / (1 - beta1^t)) m' / (sqrt(v') / sqrt(1 - beta2^t) + eps)
//
// Bound by memory: 28 bytes per element with float32 gradients and moments, 16 (14 with 16-bit gradients) with moments in
// 8 bits.  A wavefront takes units of 256 consecutive elements of a tensor, 4 per lane: every array is read and
// written in whole runs, and a unit is the block that shares a scale, so that its maximum never leaves the wavefront.
// A wavefront's kAdamUnits units are loaded before the first is used; only the last ones of a tensor are taken one by one with tests.  Which tensor a workgroup works on stands in a
// table in device memory that the caller builds once: one launch however many tensors there are, two dependent
// loads per workgroup, which the other workgroups of the compute unit hide.
// 75 M elements in 150 tensors, bf16 gradients, 8 bits: 216 to 246 us, 4.9 to 4.3 TB/s of the 5.1 that a copy reaches; the vector ALU is busy for 85 % of
// the time with three roots, a division and the roundings of every element (the compiler's full root takes 21 us more).
//
// 8 bits: m = c |c| S with a signed code c, |c| <= 127, and S = max |m| / 127^2;  sqrt(v) = c^2 S with c <= 255 and
// S = max sqrt(v) / 255^2.  Squared codes put half of the steps below a quarter of the maximum: a value of 1/100 of its
// block's maximum is held to 4 % (m) and 2 % (sqrt(v)), where equal steps hold it to 40 % and 20 %.  A positive v
// never gets the code 0: the next step would divide by eps alone.  Codes are decided by separately rounded float32
// operations.
#include "prom.h"
#include "prom_float.h"
#include "prom_launch.h"

#include <cmath>
#include <cstring>
#include <type_traits>

namespace prom {

constexpr int kAdamBlock = 256;  // elements of a unit
constexpr int kAdamUnits = 4;    // units of a wavefront
constexpr int kAdamChunk = 4 * kAdamUnits * kAdamBlock;  // elements of a workgroup of 4 wavefronts

struct AdamTensor {  // in device memory
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    long long n;
    int first;  // its first workgroup
    int8_t ptype, gtype, ctype, bits;
};
static_assert(sizeof(AdamTensor) == 72, "the table's layout");

struct AdamHyper {
    float decay, beta1, omb1, beta2, omb2, eps, step_size, inv_root2;
    const int *step;  // dev or NULL: decay, step_size and inv_root2 are then computed from lr, wd and the betas
    const float *lr, *grad_scale;
    double lr_h, wd, b1, b2;
    int step_h;
};

// b^n by squaring; the same operations on the host and on the device
__host__ __device__ inline double power(double b, int n)
{
    double r = 1.0;
    for (; n > 0; n >>= 1) {
        if (n & 1) r = r * b;
        b = b * b;
    }
    return r;
}
__host__ __device__ inline void corrections(double lr, double wd, double b1, double b2, int t, float *decay, float *step_size, float *inv_root2)
{
    *decay = (float)(1.0 - lr * wd);
    *step_size = (float)(lr / (1.0 - power(b1, t)));
    *inv_root2 = (float)(1.0 / sqrt(1.0 - power(b2, t)));
}

// m and sqrt(v) of a lane's 4 codes
__device__ __forceinline__ void decode_moments(const int8_t *c, const uint8_t *r, float ms, float vs, float (&m)[4], float (&root)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int a = c[e], b = r[e];
        m[e] = mul_f32((float)(a * (a < 0 ? -a : a)), ms);
        root[e] = mul_f32((float)(b * b), vs);
    }
}

template <typename T> __device__ __forceinline__ void load4(const T *p, long long i, int have, float (&out)[4])
{
    Piece<T, 4> q;
    q.load_some((const Global<T> *)p + i, have);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (float)q.e[e];
}
template <typename T> __device__ __forceinline__ void store4(T *p, long long i, int have, const float (&v)[4])
{
    Piece<T, 4> q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q.e[e] = (T)v[e];
    q.store_some((Global<T> *)p + i, have);
}

struct AdamScalars {
    float decay, step_size, inv_root2, grad_scale;
};

// The units of a wavefront from element `base` on; WHOLE: all of them lie in the tensor.
template <int BITS, bool WHOLE, typename TP, typename TG>
__device__ __forceinline__ void adam_units(const AdamTensor &t, const AdamHyper &h, const AdamScalars &k, long long base, int lane)
{
    constexpr int U = WHOLE ? kAdamUnits : 1;
    for (int u0 = 0; u0 < kAdamUnits; u0 += U) {
        const long long at = base + u0 * kAdamBlock;
        if (!WHOLE && at >= t.n) return;
        const int have = WHOLE ? 4 : (int)min(t.n - at - 4 * lane, 4LL);
        float p[U][4], g[U][4], m[U][4], v[U][4];
        Piece<int8_t, 4> mc[U];
        Piece<uint8_t, 4> vc[U];
        float ms[U], vs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = at + u * kAdamBlock + 4 * lane;
            load4(static_cast<const TG *>(t.g), i, have, g[u]);
            if constexpr (BITS == 8) {
                mc[u].load_some((const Global<int8_t> *)t.m + i, have);
                vc[u].load_some((const Global<uint8_t> *)t.v + i, have);
                ms[u] = ((Global<float> *)t.ms)[at / kAdamBlock + u];
                vs[u] = ((Global<float> *)t.vs)[at / kAdamBlock + u];
            } else {
                load4(static_cast<const float *>(t.m), i, have, m[u]);
                load4(static_cast<const float *>(t.v), i, have, v[u]);
            }
            load4(static_cast<const TP *>(t.p), i, have, p[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = at + u * kAdamBlock + 4 * lane;
            if constexpr (BITS == 8) {
                decode_moments(mc[u].e, vc[u].e, ms[u], vs[u], m[u], v[u]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = mul_f32(v[u][e], v[u][e]);
            }
            float root[4];
            bool small = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ge = mul_f32(g[u][e], k.grad_scale);
                m[u][e] = add_f32(mul_f32(m[u][e], h.beta1), mul_f32(ge, h.omb1));
                v[u][e] = add_f32(mul_f32(v[u][e], h.beta2), mul_f32(mul_f32(ge, h.omb2), ge));
                small |= v[u][e] < 0x1p-96f && v[u][e] > 0.0f;
            }
            if (__ballot(small)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) root[e] = sqrt_f32(v[u][e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) root[e] = sqrt_large_f32(v[u][e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float denom = add_f32(mul_f32(root[e], k.inv_root2), h.eps);
                p[u][e] = sub_f32(mul_f32(p[u][e], k.decay), __fdiv_rn(mul_f32(m[u][e], k.step_size), denom));
            }
            store4(static_cast<TP *>(t.p), i, have, p[u]);
            if (t.copy) {
                if (t.ctype == PROM_BF16) store4(static_cast<bf16_t *>(t.copy), i, have, p[u]);
                else if (t.ctype == PROM_F16) store4(static_cast<f16_t *>(t.copy), i, have, p[u]);
                else store4(static_cast<float *>(t.copy), i, have, p[u]);
            }
            if constexpr (BITS == 32) {
                store4(static_cast<float *>(t.m), i, have, m[u]);
                store4(static_cast<float *>(t.v), i, have, v[u]);
            } else {
                float mt = 0.0f, vt = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < have) {
                        mt = bits_max(mt, fabsf(m[u][e]));
                        vt = bits_max(vt, fabsf(root[e]));
                    }
                mt = wave_max_bits(mt);
                vt = wave_max_bits(vt);
                // below 2^-100 the inverse could overflow: such a block is held as zeros.  An infinity or a NaN makes the
                // scale NaN, and with it every moment of the block from the next step on, as it would in 32 bits for its element.
                constexpr float tiny = 0x1p-100f, huge = 0x1.fffffep127f;
                const float minv = mt < tiny ? 0.0f : __fdiv_rn(16129.0f, mt), vinv = vt < tiny ? 0.0f : __fdiv_rn(65025.0f, vt);
                const bool mfine = mt <= huge, vfine = vt <= huge;
                Piece<int8_t, 4> co;
                Piece<uint8_t, 4> ro;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (the root of a smaller argument than 2^-96 rounds to 0 however exact it is)
                    const float c = fminf(rintf(sqrt_large_f32(mul_f32(fabsf(m[u][e]), minv))), 127.0f);
                    float r = fminf(rintf(sqrt_large_f32(mul_f32(root[e], vinv))), 255.0f);
                    r = root[e] > 0.0f && vinv > 0.0f ? fmaxf(r, 1.0f) : r;
                    co.e[e] = mfine ? (int8_t)(m[u][e] < 0.0f ? -(int)c : (int)c) : (int8_t)0;
                    ro.e[e] = vfine ? (uint8_t)(int)r : (uint8_t)0;
                }
                co.store_some((Global<int8_t> *)t.m + i, have);
                ro.store_some((Global<uint8_t> *)t.v + i, have);
                if (lane == 0) {
                    const float nan = __int_as_float(0x7fc00000);
                    ((Global<float> *)t.ms)[at / kAdamBlock + u] = !mfine ? nan : mt < tiny ? 0.0f : mul_f32(mt, 1.0f / 16129.0f);
                    ((Global<float> *)t.vs)[at / kAdamBlock + u] = !vfine ? nan : vt < tiny ? 0.0f : mul_f32(vt, 1.0f / 65025.0f);
                }
            }
        }
    }
}

template <typename F> __device__ __forceinline__ void by_type(int type, F f)
{
    if (type == PROM_F32) f(float{});
    else if (type == PROM_BF16) f(bf16_t{});
    else f(f16_t{});
}

__global__ __launch_bounds__(256) void adamw_kernel(const AdamTensor *__restrict__ tensors, const int *__restrict__ owner, const AdamHyper h)
{
    const AdamTensor t = tensors[owner[blockIdx.x]];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long base = (long long)((int)blockIdx.x - t.first) * kAdamChunk + wave * kAdamUnits * kAdamBlock;
    if (base >= t.n) return;
    AdamScalars k{h.decay, h.step_size, h.inv_root2, h.grad_scale ? *h.grad_scale : 1.0f};
    if (h.step || h.lr) corrections(h.lr ? (double)*h.lr : h.lr_h, h.wd, h.b1, h.b2, h.step ? *h.step : h.step_h, &k.decay, &k.step_size, &k.inv_root2);
    const bool whole = base + kAdamUnits * kAdamBlock <= t.n;
    by_type(t.ptype, [&](auto tp) {
        by_type(t.gtype, [&](auto tg) {
            using TP = decltype(tp);
            using TG = decltype(tg);
            if (t.bits == 8) {
                if (whole) adam_units<8, true, TP, TG>(t, h, k, base, lane);
                else adam_units<8, false, TP, TG>(t, h, k, base, lane);
            } else {
                if (whole) adam_units<32, true, TP, TG>(t, h, k, base, lane);
                else adam_units<32, false, TP, TG>(t, h, k, base, lane);
            }
        });
    });
}

// The moments of every tensor in float32: what a checkpoint holds.
__global__ __launch_bounds__(256) void adamw_moments_kernel(const AdamTensor *__restrict__ tensors, const int *__restrict__ owner,
                                                            float *const *__restrict__ m_out, float *const *__restrict__ v_out)
{
    const int id = owner[blockIdx.x];
    const AdamTensor t = tensors[id];
    float *mo = m_out[id], *vo = v_out[id];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long base = (long long)((int)blockIdx.x - t.first) * kAdamChunk + wave * kAdamUnits * kAdamBlock;
    if (base >= t.n) return;
    auto units = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int U = WHOLE ? kAdamUnits : 1;
        for (int u0 = 0; u0 < kAdamUnits; u0 += U) {
            const long long at = base + u0 * kAdamBlock;
            if (!WHOLE && at >= t.n) return;
            const int have = WHOLE ? 4 : (int)min(t.n - at - 4 * lane, 4LL);
            float m[U][4], v[U][4];
            if (t.bits == 8) {
                Piece<int8_t, 4> mc[U];
                Piece<uint8_t, 4> vc[U];
                float ms[U], vs[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long i = at + u * kAdamBlock + 4 * lane;
                    mc[u].load_some((const Global<int8_t> *)t.m + i, have);
                    vc[u].load_some((const Global<uint8_t> *)t.v + i, have);
                    ms[u] = ((Global<float> *)t.ms)[at / kAdamBlock + u];
                    vs[u] = ((Global<float> *)t.vs)[at / kAdamBlock + u];
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    decode_moments(mc[u].e, vc[u].e, ms[u], vs[u], m[u], v[u]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[u][e] = mul_f32(v[u][e], v[u][e]);
                }
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long i = at + u * kAdamBlock + 4 * lane;
                    load4(static_cast<const float *>(t.m), i, have, m[u]);
                    load4(static_cast<const float *>(t.v), i, have, v[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long i = at + u * kAdamBlock + 4 * lane;
                store4(mo, i, have, m[u]);
                store4(vo, i, have, v[u]);
            }
        }
    };
    if (base + kAdamUnits * kAdamBlock <= t.n) units(std::true_type{});
    else units(std::false_type{});
}

// Table: [count] AdamTensor, then [chunks] int32 owners.
static long long adam_chunks(const prom_adamw_tensor_t *t, int count)
{
    long long c = 0;
    for (int i = 0; i < count; ++i) c += (t[i].n + kAdamChunk - 1) / kAdamChunk;
    return c;
}

static int adam_check(const prom_adamw_tensor_t *t, int count, int *bad)
{
    if (bad) *bad = -1;
    if (!t || count <= 0) return PROM_EINVAL;
    for (int i = 0; i < count; ++i) {
        if (bad) *bad = i;
        const prom_adamw_tensor_t &a = t[i];
        const int pb = type_bytes(a.param_type), gb = type_bytes(a.grad_type), cb = a.copy ? type_bytes(a.copy_type) : 4;
        if (!a.param || !a.grad || !a.exp_avg || !a.exp_avg_sq || a.n <= 0 || !pb || !gb || !cb) return PROM_EINVAL;
        if (a.state_bits != 8 && a.state_bits != 32) return PROM_EINVAL;
        if (a.state_bits == 8 && (!a.avg_scale || !a.sq_scale)) return PROM_EINVAL;
        const int sb = a.state_bits / 8;
        if (misaligned(a.param, pb) || misaligned(a.grad, gb) || misaligned(a.copy, cb) || misaligned(a.exp_avg, sb) || misaligned(a.exp_avg_sq, sb))
            return PROM_EINVAL;
        if (misaligned(a.avg_scale, 4) || misaligned(a.sq_scale, 4)) return PROM_EINVAL;
        if (a.n > (1LL << 42)) return PROM_EUNSUPPORTED;
        const size_t n = (size_t)a.n, blocks = a.state_bits == 8 ? (n + kAdamBlock - 1) / kAdamBlock * 4 : 0;
        const Range out[6] = {{a.param, n * pb}, {a.exp_avg, n * sb}, {a.exp_avg_sq, n * sb}, {a.copy, n * cb}, {blocks ? a.avg_scale : nullptr, blocks}, {blocks ? a.sq_scale : nullptr, blocks}};
        const Range in[1] = {{a.grad, n * gb}};
        if (outputs_meet(out, 6, in, 1)) return PROM_EALIAS;
    }
    if (bad) *bad = -1;
    if (adam_chunks(t, count) > 0xffffffLL) return PROM_EUNSUPPORTED;  // a launch has fewer than 2^32 threads
    return PROM_OK;
}

}  // namespace prom

extern "C" size_t prom_adamw_table_size(const prom_adamw_tensor_t *tensors, int count)
{
    using namespace prom;
    if (adam_check(tensors, count, nullptr) != PROM_OK) return 0;
    return sizeof(AdamTensor) * (size_t)count + 4 * (size_t)adam_chunks(tensors, count);
}

extern "C" int prom_adamw_table(const prom_adamw_tensor_t *tensors, int count, void *table_host, size_t table_bytes, prom_adamw_plan_t *plan,
                                int *bad_tensor)
{
    using namespace prom;
    if (const int rc = adam_check(tensors, count, bad_tensor)) return rc;
    if (!table_host || !plan) return PROM_EINVAL;
    const long long chunks = adam_chunks(tensors, count);
    if (table_bytes < sizeof(AdamTensor) * (size_t)count + 4 * (size_t)chunks) return PROM_EWORKSPACE;
    unsigned char *out = static_cast<unsigned char *>(table_host);
    unsigned char *owner = out + sizeof(AdamTensor) * (size_t)count;
    long long first = 0;
    for (int i = 0; i < count; ++i) {
        const prom_adamw_tensor_t &a = tensors[i];
        const AdamTensor t{a.param, a.grad, a.exp_avg, a.exp_avg_sq, a.avg_scale, a.sq_scale, a.copy, a.n, (int)first,
                           (int8_t)a.param_type, (int8_t)a.grad_type, (int8_t)a.copy_type, (int8_t)a.state_bits};
        std::memcpy(out + sizeof(AdamTensor) * (size_t)i, &t, sizeof t);
        const long long c = (a.n + kAdamChunk - 1) / kAdamChunk;
        for (long long k = 0; k < c; ++k) std::memcpy(owner + 4 * (size_t)(first + k), &i, 4);
        first += c;
    }
    plan->tensors = count;
    plan->workgroups = (int32_t)chunks;
    return PROM_OK;
}

extern "C" int prom_adamw_step(const void *table, const prom_adamw_plan_t *plan, const prom_adamw_hyper_t *h, void *stream)
{
    using namespace prom;
    if (!table || !plan || !h || plan->tensors <= 0 || plan->workgroups <= 0 || misaligned(table, 8)) return PROM_EINVAL;
    if (misaligned(h->step_dev, 4) || misaligned(h->lr_dev, 4) || misaligned(h->grad_scale, 4)) return PROM_EINVAL;
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && h->eps >= 0.0 && h->weight_decay >= 0.0)) return PROM_EINVAL;
    if (!h->step_dev && h->step < 1) return PROM_EINVAL;
    if (!h->lr_dev && !(h->lr >= 0.0)) return PROM_EINVAL;
    AdamHyper a{};
    a.beta1 = (float)h->beta1;
    a.omb1 = (float)(1.0 - h->beta1);
    a.beta2 = (float)h->beta2;
    a.omb2 = (float)(1.0 - h->beta2);
    a.eps = (float)h->eps;
    a.step = h->step_dev;
    a.lr = h->lr_dev;
    a.grad_scale = h->grad_scale;
    a.lr_h = h->lr;
    a.wd = h->weight_decay;
    a.b1 = h->beta1;
    a.b2 = h->beta2;
    a.step_h = h->step;
    if (!a.step && !a.lr) corrections(h->lr, h->weight_decay, h->beta1, h->beta2, h->step, &a.decay, &a.step_size, &a.inv_root2);
    const AdamTensor *t = static_cast<const AdamTensor *>(table);
    clear_hip_error();
    hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)plan->workgroups), dim3(256), 0, static_cast<hipStream_t>(stream), t,
                       reinterpret_cast<const int *>(t + plan->tensors), a);
    return check_launch();
}

extern "C" int prom_adamw_moments(const void *table, const prom_adamw_plan_t *plan, float *const *exp_avg, float *const *exp_avg_sq, void *stream)
{
    using namespace prom;
    if (!table || !plan || plan->tensors <= 0 || plan->workgroups <= 0 || misaligned(table, 8)) return PROM_EINVAL;
    if (!exp_avg || !exp_avg_sq || misaligned(exp_avg, 8) || misaligned(exp_avg_sq, 8)) return PROM_EINVAL;
    const AdamTensor *t = static_cast<const AdamTensor *>(table);
    clear_hip_error();
    hipLaunchKernelGGL(adamw_moments_kernel, dim3((unsigned)plan->workgroups), dim3(256), 0, static_cast<hipStream_t>(stream), t,
                       reinterpret_cast<const int *>(t + plan->tensors), exp_avg, exp_avg_sq);
    return check_launch();
}
