// Layer norm over the rows of a matrix, its gradients, and the form whose rows leave as int8 with one step each
// (the activation quantisation of paper Section 3.1, Eq. 6-7, per row), ready for the ternary pointwise layers.
//
//   mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps),  y = ((x - mean) * rstd) * weight + bias
//   g = dy * weight, h = (x - mean) * rstd:  dx = rstd * (g - sum_c g / C - h * sum_c (g h) / C)
//   dweight = sum_rows dy * h,  dbias = sum_rows dy
//
// All three are bound by the bytes of their rows.  A row is read once and stays in registers: WPR wavefronts own it, NV
// pieces of 16 bytes per lane, so that every load of a row is in flight at once and the moments, which need the
// whole row before the first output, cost no second read.  The sum of squares is taken around the mean (the row is
// there), never as a difference of large sums.  Measured: 1 x 4096 in f16 3.2 us (latency), 2048 x 2048 bf16 into int8 8.9 us
// (1.5 TB/s: two wavefronts on a SIMD, and three reductions in a row, two of them in 64 bits).
#include "prom.h"
#include "prom_float.h"
#include "prom_launch.h"

#include <type_traits>

namespace prom {

constexpr int kNormWaves = 4;  // wavefronts of a workgroup that splits rows of up to 4 wavefronts
constexpr int norm_threads(int wpr) { return 64 * (wpr > kNormWaves ? wpr : kNormWaves); }

// Sum over the WPR wavefronts of a row; part: WPR slots of the row's own, not written again before the next barrier.
template <int WPR, typename F> __device__ __forceinline__ F row_sum(F v, F *part, int wv)
{
    if constexpr (WPR == 1) return v;
    if ((threadIdx.x & 63) == 0) part[wv] = v;
    __syncthreads();
    F s = part[0];
#pragma unroll
    for (int i = 1; i < WPR; ++i) s += part[i];
    return s;
}

template <typename T, int NV, int WPR> struct NormGeom {
    static constexpr int VE = 16 / sizeof(T);  // elements of a piece
    static constexpr int WAVES = norm_threads(WPR) / 64;
    static constexpr int ROWS = WAVES / WPR;   // rows of a workgroup
};

// `have` columns from c0 on are inside the row; v: what an absent vector stands for
template <int VE> __device__ __forceinline__ void load_vector(Piece<float, VE> &p, const float *from, int c0, int have, float v)
{
    if (from) p.load_some(from + c0, have);
    else
#pragma unroll
        for (int e = 0; e < VE; ++e) p.e[e] = v;
}

struct NormArgs {
    const void *x;
    const float *weight, *bias;
    void *y;  // rows of x's type, or int8
    float *mean, *rstd, *step;
    long long rows;
    int cols;
    float eps, quant_eps;
};

// QUANT: the moments are summed in 64 bits and y is formed by separately rounded float32 operations, so that a code
// never depends on the order of a sum; 4 double operations per element, hidden behind the row's loads.
template <typename T, int NV, int WPR, bool QUANT>
__global__ __launch_bounds__(norm_threads(WPR)) void norm_kernel(const NormArgs a)
{
    using G = NormGeom<T, NV, WPR>;
    using F = typename std::conditional<QUANT, double, float>::type;
    constexpr int VE = G::VE;
    __shared__ F part[2][G::WAVES];
    __shared__ float parta[G::WAVES];
    const int lane = threadIdx.x & 63;
    const int wave = threadIdx.x >> 6;
    const int wv = wave % WPR, slot = wave / WPR;
    const long long mine = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * G::ROWS + slot;
    const bool live = mine < a.rows;
    const long long row = live ? mine : a.rows - 1;  // a wavefront without a row repeats the last one and writes nothing
    const int C = a.cols;
    const T *x = static_cast<const T *>(a.x) + row * C;

    Piece<T, VE> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
        v[i].load_some(x + c0, C - c0);
    }
    F s = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) s += (F)(float)v[i].e[e];
    if constexpr (QUANT) s = wave_sum_f64(s);
    else s = wave_sum_f32(s);
    const F mean = row_sum<WPR>(s, part[0] + slot * WPR, wv) / (F)C;
    F q = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int have = C - ((i * WPR + wv) * 64 + lane) * VE;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const F d = (F)(float)v[i].e[e] - mean;
            q += e < have ? d * d : (F)0;
        }
    }
    if constexpr (QUANT) q = wave_sum_f64(q);
    else q = wave_sum_f32(q);
    const F var = row_sum<WPR>(q, part[1] + slot * WPR, wv) / (F)C;
    const float m32 = (float)mean;
    float r32;
    if constexpr (QUANT) r32 = (float)(1.0 / sqrt(var + (double)a.eps));
    else r32 = __fdiv_rn(1.0f, sqrt_f32(var + a.eps));
    if (live && wv == 0 && lane == 0) {
        if (a.mean) a.mean[row] = m32;
        if (a.rstd) a.rstd[row] = r32;
    }

    float top = 0.0f;
    float z[QUANT ? NV : 1][VE];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
        Piece<float, VE> w, b;
        load_vector<VE>(w, a.weight, c0, C - c0, 1.0f);
        load_vector<VE>(b, a.bias, c0, C - c0, 0.0f);
        Piece<T, VE> o;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float y = add_f32(mul_f32(mul_f32(sub_f32((float)v[i].e[e], m32), r32), w.e[e]), b.e[e]);
            if constexpr (QUANT) {
                z[i][e] = y;
                if (e < C - c0) top = bits_max(top, fabsf(y));
            } else
                o.e[e] = (T)y;
        }
        if constexpr (!QUANT)
            if (live) o.store_some(static_cast<T *>(a.y) + row * C + c0, C - c0);
    }
    if constexpr (QUANT) {
        top = wave_max_bits(top);
        if constexpr (WPR > 1) {
            if (lane == 0) parta[wave] = top;
            __syncthreads();
            top = parta[slot * WPR];
#pragma unroll
            for (int i = 1; i < WPR; ++i) top = bits_max(top, parta[slot * WPR + i]);
        }
        if (top < a.quant_eps) top = a.quant_eps;  // (a NaN stays one)
        const float scale = __fdiv_rn(127.0f, top);
        if (live && wv == 0 && lane == 0) a.step[row] = __fdiv_rn(top, 127.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
            Piece<int8_t, VE> o;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                // (the clamp turns a NaN into a code; the step of such a row says that it means nothing)
                const float r = fminf(fmaxf(rintf(mul_f32(z[i][e], scale)), -128.0f), 127.0f);
                o.e[e] = (int8_t)(int)r;
            }
            if (live) o.store_some(static_cast<int8_t *>(a.y) + row * C + c0, C - c0);
        }
    }
}

// ---- gradients -----------------------------------------------------------------------------------------
// A workgroup of 16 wavefronts takes every gridDim.x-th group of rows and keeps its sums for dweight and dbias in registers from row
// to row (each lane owns its columns in all of them); they meet in LDS once at the end and leave as one row of
// partial sums per workgroup.  A second kernel adds the rows up in their order: no atomics, the same bits every time.
// The next row is on its way while one is worked on (up to two pieces a lane; more of them fill the registers).
// 8192 x 4096 bf16: 38.4 us and 5.2 for the sums where the rows still lie in the last-level cache, 48.4 and 5.4 from memory, 4.4 TB/s (with 4
// wavefronts of whole rows, 8 pieces a lane and no row ahead 117 us).
struct NormGradArgs {
    const void *dy, *x;
    const float *weight, *mean, *rstd;
    void *dx;
    float *part;  // [gridDim.x][2][cols]
    long long rows;
    int cols, want;  // want: whether dweight or dbias is asked for
};

constexpr int kNormGradWaves = 16;

template <typename T, int NV, int WPR>
__global__ __launch_bounds__(64 * kNormGradWaves) void norm_grad_kernel(const NormGradArgs a)
{
    constexpr int VE = 16 / sizeof(T);
    constexpr int ROWS = kNormGradWaves / WPR;
    __shared__ float part[2][2][kNormGradWaves];
    extern __shared__ float sums[];  // [2][columns of a row's registers] when ROWS > 1
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wv = wave % WPR, slot = wave / WPR;
    const int C = a.cols;
    const float inv = 1.0f / (float)C;
    const bool full = C == 64 * VE * NV * WPR;  // every lane has all of its columns

    float dw[NV][VE], db[NV][VE];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) dw[i][e] = db[i][e] = 0.0f;

    auto all_rows = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        auto load = [&](long long r, Piece<T, VE>(&xv)[NV], Piece<T, VE>(&gv)[NV], float &m, float &rs) __attribute__((always_inline)) {
            const T *x = static_cast<const T *>(a.x) + r * C;
            const T *dy = static_cast<const T *>(a.dy) + r * C;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
                xv[i].load_some(x + c0, WHOLE ? VE : C - c0);
                gv[i].load_some(dy + c0, WHOLE ? VE : C - c0);
            }
            m = a.mean[r];
            rs = a.rstd[r];
        };
        const long long by = (long long)gridDim.x * ROWS;
        long long r0 = (long long)blockIdx.x * ROWS;
        constexpr bool AHEAD = NV <= 2;
        Piece<T, VE> xn[NV], gn[NV];
        float mn, rn;
        if constexpr (AHEAD) load(min(r0 + slot, a.rows - 1), xn, gn, mn, rn);
        int turn = 0;
        for (; r0 < a.rows; r0 += by) {
            const bool live = r0 + slot < a.rows;
            const long long row = live ? r0 + slot : a.rows - 1;
            Piece<T, VE> xv[NV], gv[NV];
            float m, rs;
            if constexpr (AHEAD) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    xv[i] = xn[i];
                    gv[i] = gn[i];
                }
                m = mn;
                rs = rn;
                if (r0 + by < a.rows) load(min(r0 + by + slot, a.rows - 1), xn, gn, mn, rn);
            } else
                load(row, xv, gv, m, rs);
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
                Piece<float, VE> w;
                load_vector<VE>(w, a.weight, c0, WHOLE ? VE : C - c0, 1.0f);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float d = (float)gv[i].e[e];
                    const float h = ((float)xv[i].e[e] - m) * rs;
                    const bool in = WHOLE || e < C - c0;
                    if (in && live) {
                        dw[i][e] += d * h;
                        db[i][e] += d;
                    }
                    const float g = d * w.e[e];
                    s1 += in ? g : 0.0f;
                    s2 += in ? g * h : 0.0f;
                }
            }
            if (!a.dx) continue;
            s1 = wave_sum_f32(s1);
            s2 = wave_sum_f32(s2);
            if constexpr (WPR > 1) {
                // (two sets of slots in turn: one barrier per row, and one that leaves the next row's loads on their way)
                float *p1 = &part[turn & 1][0][slot * WPR], *p2 = &part[turn & 1][1][slot * WPR];
                if (lane == 0) {
                    p1[wv] = s1;
                    p2[wv] = s2;
                }
                lds_only_barrier();
                s1 = p1[0];
                s2 = p2[0];
#pragma unroll
                for (int i = 1; i < WPR; ++i) {
                    s1 += p1[i];
                    s2 += p2[i];
                }
                ++turn;
            }
            const float c1 = s1 * inv, c2 = s2 * inv;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
                Piece<float, VE> w;
                load_vector<VE>(w, a.weight, c0, WHOLE ? VE : C - c0, 1.0f);
                Piece<T, VE> o;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float h = ((float)xv[i].e[e] - m) * rs;
                    o.e[e] = (T)(((float)gv[i].e[e] * w.e[e] - c1 - h * c2) * rs);
                }
                if (live) o.store_some(static_cast<T *>(a.dx) + row * C + c0, WHOLE ? VE : C - c0);
            }
        }
    };
    if (full) all_rows(std::true_type{});
    else all_rows(std::false_type{});

    if (!a.want) return;
    float *out = a.part + (size_t)blockIdx.x * 2 * C;
    // the groups of wavefronts one after the other through LDS, the last one to memory
    for (int k = 0; k < ROWS; ++k) {
        if (k) __syncthreads();
        if (slot == k) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c0 = ((i * WPR + wv) * 64 + lane) * VE;
                Piece<float, VE> w, b;
                float *s = sums + (i * VE * WPR + wv) * 64 + lane;  // element e: 64 * WPR further each, one bank per lane
                constexpr int B = NV * VE * WPR * 64;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    w.e[e] = k ? s[e * WPR * 64] + dw[i][e] : dw[i][e];
                    b.e[e] = k ? s[e * WPR * 64 + B] + db[i][e] : db[i][e];
                    if (k < ROWS - 1) {
                        s[e * WPR * 64] = w.e[e];
                        s[e * WPR * 64 + B] = b.e[e];
                    }
                }
                if (k == ROWS - 1) {
                    w.store_some(out + c0, C - c0);
                    b.store_some(out + C + c0, C - c0);
                }
            }
        }
    }
}

// Column sums of the partial rows: 64 columns per workgroup, 4 per lane, 16 slices of the rows, then the slices.
__global__ __launch_bounds__(256) void norm_grad_sum_kernel(const float *__restrict__ part, int parts, int cols,
                                                            float *__restrict__ dweight, float *__restrict__ dbias)
{
    __shared__ v4f s[16][16];
    const int q = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int c = blockIdx.x * 64 + 4 * q;
    v4f v = {0, 0, 0, 0};
    if (c + 4 <= 2 * cols) {
#pragma unroll 8
        for (int p = slice; p < parts; p += 16) {
            Piece<float, 4> x;
            x.load(part + (size_t)p * 2 * cols + c);
            v += v4f{x.e[0], x.e[1], x.e[2], x.e[3]};
        }
    } else if (c < 2 * cols) {
        for (int p = slice; p < parts; p += 16)
            for (int e = 0; e < 4; ++e)
                if (c + e < 2 * cols) v[e] += part[(size_t)p * 2 * cols + c + e];
    }
    s[slice][q] = v;
    __syncthreads();
    if (slice == 0) {
#pragma unroll
        for (int k = 1; k < 16; ++k) v += s[k][q];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e < cols) {
                if (dweight) dweight[c + e] = v[e];
            } else if (c + e < 2 * cols && dbias)
                dbias[c + e - cols] = v[e];
        }
    }
}

// ---- launch ----------------------------------------------------------------------------------------------
constexpr int kNormMaxCols = 32768;
constexpr int kNormParts = 256;  // workgroups of the gradient kernel: one per compute unit

// Wavefronts per row: as few as hold it in 8 pieces a lane; with fewer rows than the chip has SIMDs (1024), four, so
// that a row's loads and its arithmetic are spread out.
static int norm_wpr(long long rows, int cols, int bytes)
{
    const int held = 64 * 8 * (16 / bytes);  // columns of one wavefront
    int wpr = cols <= held ? 1 : cols <= 4 * held ? 4 : 16;
    if (wpr == 1 && rows < 1024 && cols > 64 * (16 / bytes)) wpr = 4;
    return wpr;
}
static int norm_nv(int cols, int wpr, int bytes)
{
    const int one = 64 * wpr * (16 / bytes);
    const int need = (cols + one - 1) / one;
    return need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
}

template <typename T, int NV, int WPR> static void norm_launch(const NormArgs &a, bool quant, hipStream_t st)
{
    using G = NormGeom<T, NV, WPR>;
    // (a dimension of a launch has fewer than 2^32 threads)
    const long long groups = (a.rows + G::ROWS - 1) / G::ROWS, most = 1LL << 20;
    const dim3 grid((unsigned)(groups < most ? groups : most), (unsigned)((groups + most - 1) / most)), block(64 * G::WAVES);
    if (quant) hipLaunchKernelGGL((norm_kernel<T, NV, WPR, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((norm_kernel<T, NV, WPR, false>), grid, block, 0, st, a);
}
template <typename T, int NV, int WPR> static void norm_grad_launch(const NormGradArgs &a, int parts, hipStream_t st)
{
    hipLaunchKernelGGL((norm_grad_kernel<T, NV, WPR>), dim3((unsigned)parts), dim3(64 * kNormGradWaves),
                       WPR < kNormGradWaves && a.want ? (size_t)8 * 64 * WPR * NV * (16 / sizeof(T)) : 0, st, a);
}
// f(NV, WPR) as integral constants
template <typename F> static void norm_pick(int nv, int wpr, F f)
{
    auto by_wpr = [&](auto n) {
        if (wpr == 1) f(n, std::integral_constant<int, 1>{});
        else if (wpr == 4) f(n, std::integral_constant<int, 4>{});
        else f(n, std::integral_constant<int, 16>{});
    };
    if (nv == 1) by_wpr(std::integral_constant<int, 1>{});
    else if (nv == 2) by_wpr(std::integral_constant<int, 2>{});
    else if (nv == 4) by_wpr(std::integral_constant<int, 4>{});
    else by_wpr(std::integral_constant<int, 8>{});
}
template <typename F> static void norm_type(int type, F f)
{
    if (type == PROM_F32) f(float{});
    else if (type == PROM_BF16) f(bf16_t{});
    else f(f16_t{});
}

static int norm_check(const void *x, int type, long long rows, int cols, const float *weight, const float *bias)
{
    const int bytes = type_bytes(type);
    if (!x || !bytes || rows <= 0 || cols <= 0) return PROM_EINVAL;
    if (misaligned(x, bytes) || misaligned(weight, 4) || misaligned(bias, 4)) return PROM_EINVAL;
    if (cols > kNormMaxCols || rows > 0x7fffffffLL) return PROM_EUNSUPPORTED;
    return PROM_OK;
}

static int norm_forward(const void *x, int type, long long rows, int cols, const float *weight, const float *bias, float eps, float quant_eps,
                        void *y, float *step, float *mean, float *rstd, bool quant, void *stream)
{
    if (const int rc = norm_check(x, type, rows, cols, weight, bias)) return rc;
    const int bytes = type_bytes(type);
    if (!y || (quant && (!step || !(quant_eps > 0.0f))) || !(eps >= 0.0f)) return PROM_EINVAL;
    if (misaligned(y, quant ? 1 : bytes) || misaligned(step, 4) || misaligned(mean, 4) || misaligned(rstd, 4)) return PROM_EINVAL;
    const size_t rn = (size_t)rows * 4, cn = (size_t)cols * 4;
    const Range out[4] = {{y, (size_t)rows * cols * (quant ? 1 : bytes)}, {step, rn}, {mean, rn}, {rstd, rn}};
    const Range in[3] = {{x, (size_t)rows * cols * bytes}, {weight, cn}, {bias, cn}};
    if (outputs_meet(out, 4, in, 3)) return PROM_EALIAS;
    const NormArgs a{x, weight, bias, y, mean, rstd, step, rows, cols, eps, quant_eps};
    const int wpr = norm_wpr(rows, cols, bytes), nv = norm_nv(cols, wpr, bytes);
    clear_hip_error();
    norm_type(type, [&](auto t) {
        norm_pick(nv, wpr, [&](auto n, auto w) { norm_launch<decltype(t), decltype(n)::value, decltype(w)::value>(a, quant, static_cast<hipStream_t>(stream)); });
    });
    return check_launch();
}

// Wavefronts per row of the gradient kernel: as few as hold the row in two pieces a lane, and 16 beyond that.
static int norm_grad_wpr(int cols, int bytes)
{
    const int held = 64 * 2 * (16 / bytes);
    return cols <= held ? 1 : cols <= 4 * held ? 4 : 16;
}
static int norm_grad_parts(long long rows, int cols, int bytes)
{
    const int per = kNormGradWaves / norm_grad_wpr(cols, bytes);
    const long long groups = (rows + per - 1) / per;
    return (int)(groups < kNormParts ? groups : kNormParts);
}

}  // namespace prom

extern "C" int prom_layernorm(const void *x, int type, long long rows, int cols, const float *weight, const float *bias, float eps,
                              void *y, float *mean, float *rstd, void *stream)
{
    return prom::norm_forward(x, type, rows, cols, weight, bias, eps, 1.0f, y, nullptr, mean, rstd, false, stream);
}

extern "C" int prom_layernorm_quant(const void *x, int type, long long rows, int cols, const float *weight, const float *bias, float eps,
                                    float quant_eps, int8_t *q, float *step, float *mean, float *rstd, void *stream)
{
    return prom::norm_forward(x, type, rows, cols, weight, bias, eps, quant_eps, q, step, mean, rstd, true, stream);
}

extern "C" size_t prom_layernorm_backward_workspace_size(int type, long long rows, int cols)
{
    const int bytes = prom::type_bytes(type);
    if (!bytes || rows <= 0 || cols <= 0 || cols > prom::kNormMaxCols) return 0;
    return ((size_t)prom::norm_grad_parts(rows, cols, bytes) * 8 * cols + 255) / 256 * 256;
}

extern "C" int prom_layernorm_backward(const void *dy, const void *x, int type, long long rows, int cols, const float *weight,
                                       const float *mean, const float *rstd, void *dx, float *dweight, float *dbias, void *workspace,
                                       size_t workspace_bytes, void *stream)
{
    using namespace prom;
    if (const int rc = norm_check(x, type, rows, cols, weight, nullptr)) return rc;
    const int bytes = type_bytes(type);
    if (!dy || !mean || !rstd || (!dx && !dweight && !dbias)) return PROM_EINVAL;
    if (misaligned(dy, bytes) || misaligned(dx, bytes) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dweight, 4) || misaligned(dbias, 4))
        return PROM_EINVAL;
    const bool want = dweight || dbias;
    const size_t need = want ? prom_layernorm_backward_workspace_size(type, rows, cols) : 0;
    if (want && (!workspace || workspace_bytes < need || misaligned(workspace, 256))) return PROM_EWORKSPACE;
    const size_t xn = (size_t)rows * cols * bytes, rn = (size_t)rows * 4, cn = (size_t)cols * 4;
    const Range out[4] = {{dx, xn}, {dweight, cn}, {dbias, cn}, {want ? workspace : nullptr, need}};
    const Range in[5] = {{dy, xn}, {x, xn}, {weight, cn}, {mean, rn}, {rstd, rn}};
    if (outputs_meet(out, 4, in, 5)) return PROM_EALIAS;
    const int parts = norm_grad_parts(rows, cols, bytes);
    const NormGradArgs a{dy, x, weight, mean, rstd, dx, static_cast<float *>(workspace), rows, cols, want ? 1 : 0};
    const int wpr = norm_grad_wpr(cols, bytes), nv = norm_nv(cols, wpr, bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    clear_hip_error();
    norm_type(type, [&](auto t) {
        norm_pick(nv, wpr, [&](auto n, auto w) { norm_grad_launch<decltype(t), decltype(n)::value, decltype(w)::value>(a, parts, st); });
    });
    if (want)
        hipLaunchKernelGGL(norm_grad_sum_kernel, dim3((unsigned)((2 * cols + 63) / 64)), dim3(256), 0, st, static_cast<const float *>(workspace), parts,
                           cols, dweight, dbias);
    return check_launch();
}
