// Ternary pointwise layer with low-rank adapters of many requests, forward and backward: the products with the adapters,
// the gradients of the adapters, and the entry points.  The product with the shared weights is prom_lora_gemm.hip.
#include "prom_lora.h"
#include "prom_launch.h"
#include "prom_lora_gemm.h"

#include <type_traits>

namespace prom {

// ---- rows by adapter -------------------------------------------------------------------------------------
// One workgroup per adapter (and one for the elements without): it counts the elements of lower adapters and its own,
// then writes its own in their order.  Nothing has to wait for another workgroup, and the order is the same every time.
// Tile k of an adapter whose rows start at position p has the number p / tile + adapter + k: numbers of different adapters
// never meet, since floor(a) + floor(b) + 1 >= floor(a) + ceil(b), and the unused ones are written as empty.
__global__ __launch_bounds__(1024) void lora_plan_kernel(const int *__restrict__ index, int n, int hw, int adapters, LoraPlan p)
{
    __shared__ int eq_of[16], lt_of[16];
    const int l = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = ((n + 15) / 16 + 3) & ~3;
    const int from = min(n, wave * per), to = min(n, from + per);
    auto group = [&](int id) { return id >= 0 && id < adapters ? id : adapters; };
    int eq = 0, lt = 0;
    for (int i = from; i < to; i += 256) {
        const int have = to - (i + 4 * lane);
        Piece<int, 4> v;
        v.load_some(index + i + 4 * lane, have);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int g = group(v.e[e]);
            eq += __popcll(__ballot(e < have && g == l));
            lt += __popcll(__ballot(e < have && g < l));
        }
    }
    if (lane == 0) {
        eq_of[wave] = eq;
        lt_of[wave] = lt;
    }
    __syncthreads();
    int before = 0, total = 0, lower = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        if (w < wave) before += eq_of[w];
        total += eq_of[w];
        lower += lt_of[w];
    }
    int at = lower + before;
    const unsigned long long below = (1ull << lane) - 1;
    for (int i = from; i < to; i += 256) {
        const int have = to - (i + 4 * lane);
        Piece<int, 4> v;
        v.load_some(index + i + 4 * lane, have);
        unsigned long long b[4];
        int mine = at, all = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            b[e] = __ballot(e < have && group(v.e[e]) == l);
            mine += __popcll(b[e] & below);
            all += __popcll(b[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (b[e] >> lane & 1) {
                if (hw == 1) p.rows[mine] = i + 4 * lane + e;
                p.order[mine++] = i + 4 * lane + e;
            }
        at += all;
    }
    const int first = lower * hw, count = total * hw;
    if (hw > 1) {
        __syncthreads();  // (the elements above are this workgroup's own: visible to all of it behind the barrier)
        for (int i = threadIdx.x; i < count; i += 1024) {
            const int e = i / hw;
            p.rows[first + i] = p.order[lower + e] * hw + (i - e * hw);
        }
    }
    if (threadIdx.x == 0) p.groups[l] = int2{first, count};
    auto cut = [&](int4 *out, int tile) {
        const int base = first / tile + l, end = (first + count) / tile + l + 1;
        for (int k = threadIdx.x; k < end - base; k += 1024) out[base + k] = int4{l, first + k * tile, max(0, min(tile, count - k * tile)), 0};
    };
    cut(p.tiles, p.tile);
    if (p.chunks) cut(p.chunks, p.chunk);
}

// ---- the shrinking product: rows of one adapter to `rank` numbers each -------------------------------------
// A workgroup takes up to 16 I sorted rows of one adapter; its 8 wavefronts share the channels in steps of 64, every one with all of the rows
// and ranks, and their sums meet in LDS.  Bound by the activations' bytes and, from rank 32 on, by the adapter's, which every workgroup reads
// from L2.  The backward form writes the activations of the next product on the way (dy * w_scale / 2 in bf16 planes, or for a bf16 dy
// times the row's factor in f16; a ternary code reads as +-2 there), so that dy is read once for both; the factor needs the row's largest product first,
// for which the workgroup reads its rows before that.  8192 x 4096: forward at rank 32 15.6 us (22 where x comes from memory), backward at rank 16 in bf16
// 59 us, 14 of them for the factors.
struct LoraShrinkArgs {
    const void *in;     // int8 x [m][K] or dy [m][K]
    const void *low;    // [adapters][rank][K]
    const int *rows;    // [m] in sorted order
    const int4 *tiles;
    const float *step;  // [n]
    const float *scale; // [adapters] (backward)
    const float *w_scale;
    float *out;         // [m][rank]
    float *out_step;    // backward: out * step [m][rank]
    bf16_t *planes;     // backward: [m positions][P][Kp] or NULL (f16 for a bf16 dy)
    float *down;        // with them for a bf16 dy: [m]
    int hw, K, Kp, rank, adapters;
};

// eight bf16 of eight int8 codes (exact: 8 significant bits)
__device__ __forceinline__ v8bf codes_to_bf16(const int8_t *c)
{
    v8bf r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16_t)(float)c[e];
    return r;
}

template <bool BACK, typename TX, typename TA, int RT, int I>
__global__ __launch_bounds__(512) void lora_shrink_kernel(const LoraShrinkArgs a)
{
    constexpr int PA = planes_of<TA>();
    constexpr int PX = BACK ? planes_of<TX>() : 1;  // (codes: one plane)
    constexpr bool SCALED = BACK && kScaledPlane<TX>;
    using TE = typename std::conditional<SCALED, f16_t, bf16_t>::type;
    constexpr int KS = 64, KL = 16;  // channels of a step, of them a lane's
    constexpr int BY = KS * 8;       // from one step of a wavefront to its next
    __shared__ v4f red[4][I * RT][64];
    __shared__ float widest[SCALED ? 16 * I : 1];
    const int4 tile = a.tiles[blockIdx.x];
    const int l = tile.x, count = tile.z;
    if (count == 0) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = lane & 15, g = lane >> 4;
    const bool has = l < a.adapters;
    const int K = a.K;

    int row[I], elem[I];
    bool in[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        in[i] = 16 * i + j < count;
        row[i] = a.rows[tile.y + min(16 * i + j, count - 1)];
        elem[i] = a.hw == 1 ? row[i] : row[i] / a.hw;
    }
    v4f acc[I][RT];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[i][t] = v4f{0, 0, 0, 0};

    const int end = K / KS * KS;  // whole steps
    float up[I];
    if constexpr (SCALED)
        if (a.planes) {  // the rows' largest products, 2 I rows of a wavefront whole and in runs of 1 KB
            constexpr int R = 2 * I, N = 4 / I;  // N runs' loads leave together
            if (wave * R < count) {
                const TX *from[R];
                float most[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    from[r] = static_cast<const TX *>(a.in) + (size_t)a.rows[tile.y + min(wave * R + r, count - 1)] * K;
                    most[r] = 0.0f;
                }
                auto look = [&](auto whole, int k, int u) __attribute__((always_inline)) {
                    constexpr bool WHOLE = decltype(whole)::value;
                    constexpr int M = WHOLE ? N : 1;
                    Piece<TX, 8> v[M][R];
                    Piece<float, 8> ws[M];
#pragma unroll
                    for (int n = 0; n < M; ++n) {
                        const int k0 = k + 512 * (n < u ? n : 0) + 8 * lane;
#pragma unroll
                        for (int r = 0; r < R; ++r) v[n][r].load_some_at_once(from[r] + k0, WHOLE ? 8 : K - k0);
                        ws[n].load_some(a.w_scale + k0, WHOLE ? 8 : K - k0);
                    }
#pragma unroll
                    for (int n = 0; n < M; ++n)  // (the repeated ones change nothing)
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int e = 0; e < 8; ++e) most[r] = bits_max(most[r], fabsf((float)v[n][r].e[e] * ws[n].e[e]));
                };
                const int runs = K & ~511;
                for (int k = 0; k < runs; k += 512 * N) look(std::true_type{}, k, min(N, (runs - k) >> 9));
                if (runs < K) look(std::false_type{}, runs, 1);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    most[r] = wave_max_bits(most[r]);
                    if (lane == 0) widest[wave * R + r] = most[r];
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < I; ++i) {
                up[i] = plane_up(widest[min(16 * i + j, count - 1)]);
                if (wave == 0 && g == 0 && in[i]) a.down[row[i]] = plane_down(up[i]);
            }
        }

    const TA *low = static_cast<const TA *>(a.low) + (size_t)(has ? l : 0) * a.rank * K;
    // U steps of loads leave together before the first of them is used: there are 2 to 4 wavefronts on a SIMD to wait with
    // (rank 32, 8192 x 4096: 20 us with one step at a time)
    constexpr int U = BACK ? (RT == 1 ? (PX == 1 ? 4 : 2) : RT == 2 ? 2 : 1) : RT <= 2 ? 4 : RT == 4 ? 2 : 1;
    auto steps = [&](auto whole, int k, int by, int u) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int N = WHOLE ? U : 1;
        Piece<TX, 16> v[N][I];
        Piece<float, 16> ws[N];
        Piece<TA, 8> w[N][RT][KL / 8];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int k0 = k + (n < u ? n : 0) * by + KL * g;
#pragma unroll
            for (int i = 0; i < I; ++i) v[n][i].load_some(static_cast<const TX *>(a.in) + (size_t)row[i] * K + k0, WHOLE ? 16 : K - k0);
            if (BACK && a.planes) ws[n].load_some(a.w_scale + k0, WHOLE ? 16 : K - k0);
            if (has)
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const int r = min(16 * t + j, a.rank - 1);  // (ranks past the last one repeat it and are not written)
#pragma unroll
                    for (int h = 0; h < KL / 8; ++h) w[n][t][h].load_some(low + (size_t)r * K + k0 + 8 * h, WHOLE ? 8 : K - k0 - 8 * h);
                }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (n >= u) break;
            const int k0 = k + n * by + KL * g;
            v8bf bx[I][2][PX];
            if constexpr (BACK) {
                if (a.planes) {
#pragma unroll
                    for (int i = 0; i < I; ++i) {
                        Piece<TE, 16> o[PX];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            TE s[PX];
                            const float x = (float)v[n][i].e[e] * ws[n].e[e];
                            if constexpr (SCALED) s[0] = (f16_t)(x * up[i]);
                            else split<PX>(x * 0.5f, s);
                            // (the decoded codes come in the order 0, 2, 1, 3 of every four)
                            constexpr int to[4] = {0, 2, 1, 3};
#pragma unroll
                            for (int p = 0; p < PX; ++p) o[p].e[(e & ~3) + to[e & 3]] = s[p];
                        }
                        const size_t pos = (size_t)(tile.y + 16 * i + j);
                        if (in[i])
#pragma unroll
                            for (int p = 0; p < PX; ++p) o[p].store(reinterpret_cast<TE *>(a.planes) + (pos * PX + p) * a.Kp + k0);
                    }
                }
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Piece<TX, 8> half;
#pragma unroll
                        for (int e = 0; e < 8; ++e) half.e[e] = v[n][i].e[8 * h + e];
                        split_piece<PX>(half, bx[i][h]);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    bx[i][0][0] = codes_to_bf16(v[n][i].e);
                    bx[i][1][0] = codes_to_bf16(v[n][i].e + 8);
                }
            }
            if (!has) continue;
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int h = 0; h < KL / 8; ++h) {
                    v8bf aw[PA];
                    split_piece<PA>(w[n][t][h], aw);
#pragma unroll
                    for (int i = 0; i < I; ++i) {
#pragma unroll
                        for (int p = 0; p < PA; ++p)
#pragma unroll
                            for (int q = 0; q < PX; ++q)
                                if (p + q < 3) acc[i][t] = mfma_bf16(aw[p], bx[i][h][q], acc[i][t]);
                    }
                }
        }
    };
    if (BACK || has) {
        int k = KS * wave;
        for (; k < end; k += U * BY) steps(std::true_type{}, k, BY, min(U, (end - k + BY - 1) / BY));
        // what is left behind the whole steps, and the planes' padding
        const int limit = BACK && a.planes ? a.Kp : K;
        for (k = end; k < limit; k += KS)
            if ((k / KS & 7) == wave) steps(std::false_type{}, k, 0, 1);
    }
    // sums of the 8 wavefronts, always added in the same order
    if (wave >= 4)
#pragma unroll
        for (int c = 0; c < I * RT; ++c) red[wave - 4][c][lane] = acc[c % I][c / I];
    __syncthreads();
    if (wave < 4)
#pragma unroll
        for (int c = 0; c < I * RT; ++c) {
            const v4f o = red[wave][c][lane];
            red[wave][c][lane] = acc[c % I][c / I] + o;
        }
    __syncthreads();
#pragma unroll
    for (int c0 = 0; c0 < I * RT; c0 += 8) {
        const int c = c0 + wave;
        if (c >= I * RT) break;
        const v4f s = (red[0][c][lane] + red[1][c][lane]) + (red[2][c][lane] + red[3][c][lane]);
        const int i = c % I, t = c / I;
        const bool ok = i ? in[I - 1] : in[0];
        const int r0 = i ? row[I - 1] : row[0];
        const float step = a.step[i ? elem[I - 1] : elem[0]];
        const float f = !has ? 0.0f : BACK ? a.scale[l] : step;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 16 * t + 4 * g + e;
            if (ok && r < a.rank) {
                const float v = has ? s[e] * f : 0.0f;
                a.out[(size_t)r0 * a.rank + r] = v;
                if (BACK && a.out_step) a.out_step[(size_t)r0 * a.rank + r] = v * step;
            }
        }
    }
}

// The same for fewer rows, without sorting: a wavefront per row and RC ranks, the channels over its lanes, float32 on the vector
// ALU.  Every row reads its own adapter; what bounds it is the latency of two dependent loads and, with many rows, the adapters' bytes (64 rows of
// 4096 channels, rank 16, 64 adapters: 5.9 us).
template <typename TA, int RC>
__global__ __launch_bounds__(256) void lora_shrink_small_kernel(const int8_t *__restrict__ x, const TA *__restrict__ low, const int *__restrict__ index,
                                                                const float *__restrict__ step, float *__restrict__ hid, int m, int hw, int K,
                                                                int rank, int adapters)
{
    const int lane = threadIdx.x & 63;
    const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int per = (rank + RC - 1) / RC;
    const int row = unit / per, r0 = (unit - row * per) * RC;
    if (row >= m) return;
    const int l = index[row / hw];
    const bool has = l >= 0 && l < adapters;
    float s[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) s[c] = 0.0f;
    if (has) {
        const int8_t *xr = x + (size_t)row * K;
        const TA *lr = low + ((size_t)l * rank + r0) * K;
        // U steps of 512 channels at a time: with 8 a row of 4096 channels leaves in one go
        constexpr int U = RC == 1 ? 8 : 4;
        const int end = K & ~511;
        auto steps = [&](auto whole, int k, int u) __attribute__((always_inline)) {
            constexpr bool WHOLE = decltype(whole)::value;
            constexpr int N = WHOLE ? U : 1;
            Piece<int8_t, 8> v[N];
            Piece<TA, 8> w[N][RC];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int k0 = k + 512 * (n < u ? n : 0) + 8 * lane;
                v[n].load_some(xr + k0, WHOLE ? 8 : K - k0);
#pragma unroll
                for (int c = 0; c < RC; ++c) w[n][c].load_some(lr + (size_t)(r0 + c < rank ? c : 0) * K + k0, WHOLE ? 8 : K - k0);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n >= u) break;
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int c = 0; c < RC; ++c) s[c] += (float)v[n].e[e] * (float)w[n][c].e[e];
            }
        };
        for (int k = 0; k < end; k += 512 * U) steps(std::true_type{}, k, min(U, (end - k) >> 9));
        if (end < K) steps(std::false_type{}, end, 1);
    }
    const float f = step[row / hw];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
        const float t = wave_sum_f32(s[c]);
        if (lane == 0 && r0 + c < rank) hid[(size_t)row * rank + r0 + c] = has ? t * f : 0.0f;
    }
}

// ---- gradients of the adapters ------------------------------------------------------------------------------
// out_l [rank][C] = sum over the rows of adapter l of coef [row][rank]^T times in [row][C]: both operands of the matrix
// instruction run along the rows, across the memory's order.  A lane loads 8 rows x 8 neighbouring columns and turns them in
// its own registers (pairs of rows by v_perm); it then holds 8 rows of its 8 columns, which is one operand for each of
// 8 tiles whose 16 columns lie 8 apart: no LDS, whole runs of 8 bytes (int8) or 16 to 32 a lane.  A workgroup takes 512 columns and a chunk
// of one adapter's sorted rows, and writes partial sums; a second kernel adds an adapter's chunks in their order.  8192 rows of 4096 int8
// and 4096 bf16 columns, rank 16: 38 us and 10 for the sums; bound by the latency of gathered rows, two steps ahead at most.
struct LoraGradArgs {
    const void *in;      // [m][C]
    const float *coef;   // [m][rank]
    const float *scale;  // [adapters] or NULL: factor of the coefficients
    float *part;         // [chunks][rank][C]
    float *out;          // [adapters][rank][C]
    int C, blocks;       // blocks: workgroups of 512 columns, 0: not asked for
};
struct LoraGradBoth {    // da (int8 rows) and db share a launch: alone neither fills the chip
    LoraGradArgs a, b;
    const int *rows;
    const int4 *chunks;
    const int2 *groups;
    int rank, adapters, chunk;
};

template <typename TX, int RT>
__device__ __forceinline__ void lora_grad_part(const LoraGradBoth &all, const LoraGradArgs &a, int block)
{
    constexpr bool CODES = std::is_same<TX, int8_t>::value;
    constexpr int PX = CODES ? 1 : planes_of<TX>();
    const int4 chunk = all.chunks[blockIdx.x];
    if (chunk.z == 0 || chunk.x >= all.adapters) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = lane & 15, g = lane >> 4;
    const int c0 = (block * 4 + wave) * 128 + 8 * j;
    const int r0 = blockIdx.z * 16 * RT;
    if ((block * 4 + wave) * 128 >= a.C) return;
    const float f = a.scale ? a.scale[chunk.x] : 1.0f;

    v4f acc[RT][8];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[t][e] = v4f{0, 0, 0, 0};

    // Row numbers are fetched two steps of 32 rows ahead, rows and coefficients one.  (The next step's loads behind the
    // last one repeat it: they are not used.)
    auto all_rows = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;  // every step has 32 rows and every lane 8 columns
        auto load_rows = [&](int m, Piece<int, 8> &row) __attribute__((always_inline)) {
            row.load_some(all.rows + chunk.y + m + 8 * g, WHOLE ? 8 : chunk.z - m - 8 * g);
        };
        auto load = [&](int m, const Piece<int, 8> &row, Piece<TX, 8>(&v)[8], float(&c)[RT][8]) __attribute__((always_inline)) {
            const int have = WHOLE ? 8 : chunk.z - m - 8 * g;  // rows of this lane
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e].load_some_at_once(static_cast<const TX *>(a.in) + (size_t)row.e[e] * a.C + c0, WHOLE ? 8 : e < have ? a.C - c0 : 0);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    c[t][e] = 0.0f;
                    if (e < have) c[t][e] = a.coef[(size_t)row.e[e] * all.rank + min(r0 + 16 * t + j, all.rank - 1)];
                }
            }
        };
        Piece<int, 8> row;
        Piece<TX, 8> v[8];
        float cf[RT][8];
        load_rows(0, row);
        load(0, row, v, cf);
        const int last = (chunk.z - 1) & ~31;
        load_rows(min(32, last), row);
        for (int m = 0; m < chunk.z; m += 32) {
            Piece<TX, 8> now[8];
            v8bf co[RT][3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                now[e] = v[e];
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    bf16_t s[3];
                    split<3>(cf[t][e] * f, s);
#pragma unroll
                    for (int p = 0; p < 3; ++p) co[t][p][e] = s[p];
                }
            }
            if (m < last) {
                load(m + 32, row, v, cf);
                load_rows(min(m + 64, last), row);
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                v8bf b[PX];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (CODES) b[0][e] = (bf16_t)(float)now[e].e[c];
                    else if constexpr (PX == 1) b[0][e] = now[e].e[c];
                    else {
                        bf16_t s[PX];
                        split<PX>((float)now[e].e[c], s);
#pragma unroll
                        for (int p = 0; p < PX; ++p) b[p][e] = s[p];
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int p = 0; p < 3; ++p)
#pragma unroll
                        for (int q = 0; q < PX; ++q)
                            if (p + q < 3) acc[t][c] = mfma_bf16(co[t][p], b[q], acc[t][c]);
            }
        }
    };
    const int col = (block * 4 + wave) * 128;
    if ((chunk.z & 31) == 0 && col + 128 <= a.C) all_rows(std::true_type{});
    else all_rows(std::false_type{});
    // lane (j, g), register e of tile (t, c): rank 16t + 4g + e, column c0 + c
    float *out = a.part + (size_t)blockIdx.x * all.rank * a.C;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + 16 * t + 4 * g + e;
            if (r >= all.rank) continue;
            Piece<float, 8> o;
#pragma unroll
            for (int c = 0; c < 8; ++c) o.e[c] = acc[t][c][e];
            o.store_some(out + (size_t)r * a.C + c0, a.C - c0);
        }
}

template <typename TX, int RT>
__global__ __launch_bounds__(256) void lora_grad_kernel(const LoraGradBoth all)
{
    if ((int)blockIdx.y < all.a.blocks) lora_grad_part<int8_t, RT>(all, all.a, blockIdx.y);
    else lora_grad_part<TX, RT>(all, all.b, blockIdx.y - all.a.blocks);
}

// An adapter's chunks one after the other, in 64 bits: 2^20 rows are a chain of 8192 additions, which in float32 lose up to 1400 * 2^-24 where the
// terms are alike.  Bound by the partial sums' bytes either way.
__global__ __launch_bounds__(256) void lora_grad_sum_kernel(const LoraGradBoth all)
{
    const int na = all.a.blocks ? (all.a.C + 1023) / 1024 : 0;
    const bool first = (int)blockIdx.y < na;
    const LoraGradArgs &a = first ? all.a : all.b;
    const int rank = all.rank, C = a.C;
    const int l = blockIdx.x / rank, r = blockIdx.x - l * rank;
    const int c0 = (((int)blockIdx.y - (first ? 0 : na)) * 256 + threadIdx.x) * 4;
    if (c0 >= C) return;
    const int2 grp = all.groups[l];
    const int base = grp.x / all.chunk + l, chunks = (grp.y + all.chunk - 1) / all.chunk;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (int k = 0; k < chunks; ++k) {
        Piece<float, 4> v;
        v.load_some(a.part + ((size_t)(base + k) * rank + r) * C + c0, C - c0);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += (double)v.e[e];
    }
    Piece<float, 4> o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o.e[e] = (float)s[e];
    o.store_some(a.out + ((size_t)l * rank + r) * C + c0, C - c0);
}

// ---- host -------------------------------------------------------------------------------------------------
static size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// Rows of a chunk of the adapters' gradients.  More chunks keep more loads on their way, and every one costs rank * (cin + cout) * 4 bytes of
// partial sums, written and read: 8192 x 4096 -> 4096, rank 16, both gradients with their sums 47 us with 128 rows, 47 with 256, 64 with 512;
// 500 x 1000 -> 1030 in float32 22, 29 and 29.
constexpr int kLoraChunk = 128;

template <typename F> static void by_adapter_type(int type, F f)
{
    if (type == PROM_BF16) f(bf16_t{});
    else f(f16_t{});
}
template <typename F> static void by_real_type(int type, F f)
{
    if (type == PROM_F32) f(float{});
    else by_adapter_type(type, f);
}
// Rows of a workgroup of the shrinking product.  Forward 32: every workgroup reads the adapter again, from rank 16 on as many bytes as
// its activations are (8192 x 4096, rank 32: 15.6 us, with 16 rows 22.7).  Backward 16 up to rank 32, where the
// activations are twice the bytes, written once more: more workgroups keep more of them on their way (8192 x 4096 in bf16 at
// rank 16: 59 us, with 32 rows 66; 500 x 1030 in float32 at rank 12 11.6 and 17.4).
static int lora_tile(int rank, bool back) { return back && rank <= 32 ? 16 : 32; }
// f(rank tiles of 16, row tiles of 16)
template <typename F> static void by_rank(int rank, bool back, F f)
{
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    if (rank <= 16) back ? f(One{}, One{}) : f(One{}, Two{});
    else if (rank <= 32) back ? f(Two{}, One{}) : f(Two{}, Two{});
    else if (rank <= 64) f(std::integral_constant<int, 4>{}, Two{});
    else f(std::integral_constant<int, 8>{}, Two{});
}

struct LoraSpace {  // offsets into the workspace
    size_t order, rows, groups, tiles, chunks, hid, g, gs, planes, down, part_a, part_b, bytes;
    int ntiles, nchunks;
};
static LoraSpace lora_space(long long m, int n, int cin, int cout, int adapters, int rank, bool back, int planes)
{
    LoraSpace s{};
    size_t at = 0;
    auto take = [&](size_t b) {
        const size_t o = at;
        at += up256(b);
        return o;
    };
    s.ntiles = (int)(m / lora_tile(rank, back)) + adapters + 1;
    s.nchunks = (int)(m / kLoraChunk) + adapters + 1;
    s.order = take((size_t)n * 4);
    s.rows = take((size_t)m * 4);
    s.groups = take((size_t)(adapters + 1) * 8);
    s.tiles = take((size_t)s.ntiles * 16);
    if (back) {
        s.chunks = take((size_t)s.nchunks * 16);
        s.g = take((size_t)m * rank * 4);
        s.gs = take((size_t)m * rank * 4);
        s.planes = take((size_t)m * planes * lora_padded(cout) * 2);
        s.down = take(planes == 1 ? (size_t)m * 4 : 0);
        s.part_a = take((size_t)s.nchunks * rank * cin * 4);
        s.part_b = take((size_t)s.nchunks * rank * cout * 4);
    } else
        s.hid = take((size_t)m * rank * 4);
    s.bytes = at;
    return s;
}

static int lora_check(int n, int h, int w, int cin, int cout, const prom_lora_t *lo, long long *m)
{
    if (!lo || n <= 0 || h <= 0 || w <= 0 || cin <= 0 || cout <= 0) return PROM_EINVAL;
    if (!lo->a || !lo->b || !lo->scale || !lo->index || lo->adapters <= 0 || lo->rank <= 0) return PROM_EINVAL;
    if (lo->type != PROM_BF16 && lo->type != PROM_F16) return PROM_EINVAL;
    if (misaligned(lo->a, 2) || misaligned(lo->b, 2) || misaligned(lo->scale, 4) || misaligned(lo->index, 4)) return PROM_EINVAL;
    if (cin > kLoraMaxChannels || cout > kLoraMaxChannels || lo->rank > kLoraMaxRank || lo->adapters > kLoraMaxAdapters) return PROM_EUNSUPPORTED;
    const long long hw = (long long)h * w;
    if (hw > kLoraMaxRows || hw * n > kLoraMaxRows) return PROM_EUNSUPPORTED;
    *m = hw * n;
    return PROM_OK;
}

// Up to this many rows run without sorting, on the kernels whose workgroups hold every row.
constexpr int kLoraFew = 64;

// rows * rank up to which the shrinking product of the forward call goes row by row: the tiles of sorted rows are too few to fill the chip, and the
// adapters, read once per row, still come out of L2 fast enough (4096 channels, 512 rows of rank 16 and 1000 of rank 8: 7.0 and 6.2 us, in tiles 16).
constexpr int kLoraUnsorted = 16384;

static int planes_of_type(int type) { return type == PROM_F32 ? 3 : type == PROM_F16 ? 2 : 1; }

}  // namespace prom

namespace prom {
static bool lora_sizes(int n, int h, int w, int cin, int cout, int adapters, int rank, long long *m)
{
    if (n <= 0 || h <= 0 || w <= 0 || cin <= 0 || cout <= 0 || adapters <= 0 || rank <= 0) return false;
    if (cin > kLoraMaxChannels || cout > kLoraMaxChannels || rank > kLoraMaxRank || adapters > kLoraMaxAdapters) return false;
    const long long hw = (long long)h * w;
    if (hw > kLoraMaxRows || hw * n > kLoraMaxRows) return false;
    *m = hw * n;
    return true;
}
// Bytes the forward call looks at.
static size_t lora_forward_bytes(long long m, const LoraSpace &s, bool has_hid) { return m <= kLoraFew && has_hid ? 0 : s.bytes; }
}  // namespace prom

extern "C" size_t prom_pw_conv_lora_workspace_size(int n, int h, int w, int cin, int cout, int adapters, int rank, int has_hid)
{
    using namespace prom;
    long long m = 0;
    if (!lora_sizes(n, h, w, cin, cout, adapters, rank, &m)) return 0;
    return lora_forward_bytes(m, lora_space(m, n, cin, cout, adapters, rank, false, 0), has_hid != 0);
}

extern "C" int prom_pw_conv_lora(const int8_t *x, int n, int h, int w, int cin, const void *w_packed, int cout, const float *x_step,
                                 const float *w_scale, const float *bias, const prom_lora_t *lora, void *y, int y_type, float *hid, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    using namespace prom;
    long long m = 0;
    if (!w_packed || misaligned(w_packed, 4)) return PROM_EINVAL;
    if (const int rc = lora_check(n, h, w, cin, cout, lora, &m)) return rc;
    if (!x || !x_step || !w_scale || !y || (y_type != PROM_F32 && y_type != lora->type)) return PROM_EINVAL;
    const int yb = type_bytes(y_type);
    if (misaligned(x_step, 4) || misaligned(w_scale, 4) || misaligned(bias, 4) || misaligned(y, yb) || misaligned(hid, 4)) return PROM_EINVAL;
    const LoraSpace s = lora_space(m, n, cin, cout, lora->adapters, lora->rank, false, 0);
    const size_t need = lora_forward_bytes(m, s, hid != nullptr);
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 256))) return PROM_EWORKSPACE;
    const size_t pool = (size_t)lora->adapters * lora->rank * 2;
    const Range out[3] = {{y, (size_t)m * cout * yb}, {hid, (size_t)m * lora->rank * 4}, {need ? workspace : nullptr, need}};
    const Range in[9] = {{x, (size_t)m * cin}, {w_packed, prom_packed_size(cout, cin)}, {x_step, (size_t)n * 4}, {w_scale, (size_t)cout * 4},
                         {bias, (size_t)cout * 4}, {lora->a, pool * cin}, {lora->b, pool * cout}, {lora->scale, (size_t)lora->adapters * 4},
                         {lora->index, (size_t)n * 4}};
    if (outputs_meet(out, 3, in, 9)) return PROM_EALIAS;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    if (!hid) hid = reinterpret_cast<float *>(ws + s.hid);
    LoraGemmArgs ga{};
    ga.x = x;
    ga.wq = static_cast<const uint32_t *>(w_packed);
    ga.index = lora->index;
    ga.step = x_step;
    ga.w_scale = w_scale;
    ga.bias = bias;
    ga.hid = hid;
    ga.scale = lora->scale;
    ga.low = lora->b;
    ga.y = y;
    ga.m = (int)m;
    ga.hw = h * w;
    ga.K = cin;
    ga.KW = (cin + 15) / 16;
    ga.Nc = cout;
    ga.rank = lora->rank;
    ga.adapters = lora->adapters;
    clear_hip_error();
    // Every row with its own adapter, without sorting: a rank per wavefront while that leaves SIMDs idle, four (which share the row's codes) from then on.
    auto shrink_small = [&]() {
        by_adapter_type(lora->type, [&](auto t) {
            using T = decltype(t);
            auto go = [&](auto rc) {
                constexpr int RC = decltype(rc)::value;
                const long long units = m * ((lora->rank + RC - 1) / RC);
                hipLaunchKernelGGL((lora_shrink_small_kernel<T, RC>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st, x, static_cast<const T *>(lora->a),
                                   lora->index, x_step, hid, (int)m, ga.hw, cin, lora->rank, lora->adapters);
            };
            if (m * lora->rank <= 1024) go(std::integral_constant<int, 1>{});
            else go(std::integral_constant<int, 4>{});
        });
    };
    if (m <= kLoraFew) {
        if (m * lora->rank <= kFuseMost) {
            ga.first = lora->a;
            ga.hid_out = hid;
        } else
            shrink_small();
        lora_gemm_few(ga, lora->type, y_type, st);
        return check_launch();
    }
    LoraPlan p{};
    p.order = reinterpret_cast<int *>(ws + s.order);
    p.rows = reinterpret_cast<int *>(ws + s.rows);
    p.groups = reinterpret_cast<int2 *>(ws + s.groups);
    p.tiles = reinterpret_cast<int4 *>(ws + s.tiles);
    p.tile = lora_tile(lora->rank, false);
    hipLaunchKernelGGL(lora_plan_kernel, dim3((unsigned)lora->adapters + 1), dim3(1024), 0, st, lora->index, n, ga.hw, lora->adapters, p);
    LoraShrinkArgs sa{};
    sa.in = x;
    sa.low = lora->a;
    sa.rows = p.rows;
    sa.tiles = p.tiles;
    sa.step = x_step;
    sa.out = hid;
    sa.hw = ga.hw;
    sa.K = cin;
    sa.rank = lora->rank;
    sa.adapters = lora->adapters;
    if (m * lora->rank <= kLoraUnsorted) shrink_small();
    else by_adapter_type(lora->type, [&](auto t) {
        by_rank(lora->rank, false, [&](auto rt, auto it) {
            hipLaunchKernelGGL((lora_shrink_kernel<false, int8_t, decltype(t), decltype(rt)::value, decltype(it)::value>), dim3((unsigned)s.ntiles), dim3(512), 0, st, sa);
        });
    });
    ga.rows = p.rows;
    lora_gemm(ga, lora->type, y_type, false, st);
    return check_launch();
}

extern "C" size_t prom_pw_conv_lora_backward_workspace_size(int n, int h, int w, int cin, int cout, int adapters, int rank, int dy_type)
{
    using namespace prom;
    long long m = 0;
    if (!lora_sizes(n, h, w, cin, cout, adapters, rank, &m) || !type_bytes(dy_type)) return 0;
    return lora_space(m, n, cin, cout, adapters, rank, true, planes_of_type(dy_type)).bytes;
}

extern "C" int prom_pw_conv_lora_backward(const void *dy, int dy_type, const int8_t *x, int n, int h, int w, int cin, const void *wt_packed, int cout,
                                          const float *x_step, const float *w_scale, const prom_lora_t *lora, const float *hid, void *dx, float *da,
                                          float *db, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace prom;
    long long m = 0;
    if (dx && (!wt_packed || misaligned(wt_packed, 4))) return PROM_EINVAL;
    if (const int rc = lora_check(n, h, w, cin, cout, lora, &m)) return rc;
    if (!dy || !x_step || (!dx && !da && !db) || (dx && !w_scale) || (da && !x) || (db && !hid)) return PROM_EINVAL;
    if (dy_type != PROM_F32 && dy_type != lora->type) return PROM_EINVAL;
    const int yb = type_bytes(dy_type), planes = planes_of_type(dy_type);
    if (misaligned(dy, yb) || misaligned(dx, yb) || misaligned(x_step, 4) || misaligned(w_scale, 4) || misaligned(hid, 4) || misaligned(da, 4) || misaligned(db, 4))
        return PROM_EINVAL;
    const LoraSpace s = lora_space(m, n, cin, cout, lora->adapters, lora->rank, true, planes);
    if (!workspace || workspace_bytes < s.bytes || misaligned(workspace, 256)) return PROM_EWORKSPACE;
    const size_t pool = (size_t)lora->adapters * lora->rank;
    const Range out[4] = {{dx, (size_t)m * cin * yb}, {da, pool * cin * 4}, {db, pool * cout * 4}, {workspace, s.bytes}};
    const Range in[9] = {{dy, (size_t)m * cout * yb}, {x, (size_t)m * cin}, {dx ? wt_packed : nullptr, prom_packed_size(cin, cout)}, {x_step, (size_t)n * 4},
                         {w_scale, (size_t)cout * 4}, {lora->a, pool * cin * 2}, {lora->b, pool * cout * 2}, {hid, (size_t)m * lora->rank * 4},
                         {lora->index, (size_t)n * 4}};
    const Range more[1] = {{lora->scale, (size_t)lora->adapters * 4}};
    if (outputs_meet(out, 4, in, 9) || outputs_meet(out, 4, more, 1)) return PROM_EALIAS;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    const int hw = h * w;
    LoraPlan p{};
    p.order = reinterpret_cast<int *>(ws + s.order);
    p.rows = reinterpret_cast<int *>(ws + s.rows);
    p.groups = reinterpret_cast<int2 *>(ws + s.groups);
    p.tiles = reinterpret_cast<int4 *>(ws + s.tiles);
    p.tile = lora_tile(lora->rank, true);
    p.chunks = reinterpret_cast<int4 *>(ws + s.chunks);
    p.chunk = kLoraChunk;
    clear_hip_error();
    hipLaunchKernelGGL(lora_plan_kernel, dim3((unsigned)lora->adapters + 1), dim3(1024), 0, st, lora->index, n, hw, lora->adapters, p);
    LoraShrinkArgs sa{};
    sa.in = dy;
    sa.low = lora->b;
    sa.rows = p.rows;
    sa.tiles = p.tiles;
    sa.step = x_step;
    sa.scale = lora->scale;
    sa.w_scale = w_scale;
    sa.out = reinterpret_cast<float *>(ws + s.g);
    sa.out_step = reinterpret_cast<float *>(ws + s.gs);
    sa.planes = dx ? reinterpret_cast<bf16_t *>(ws + s.planes) : nullptr;
    sa.down = reinterpret_cast<float *>(ws + s.down);
    sa.hw = hw;
    sa.K = cout;
    sa.Kp = lora_padded(cout);
    sa.rank = lora->rank;
    sa.adapters = lora->adapters;
    by_adapter_type(lora->type, [&](auto t) {
        by_rank(lora->rank, true, [&](auto rt, auto it) {
            const dim3 grid((unsigned)s.ntiles), block(512);
            if (dy_type == PROM_F32)
                hipLaunchKernelGGL((lora_shrink_kernel<true, float, decltype(t), decltype(rt)::value, decltype(it)::value>), grid, block, 0, st, sa);
            else
                hipLaunchKernelGGL((lora_shrink_kernel<true, decltype(t), decltype(t), decltype(rt)::value, decltype(it)::value>), grid, block, 0, st, sa);
        });
    });
    if (dx) {
        LoraGemmArgs ga{};
        ga.x = ws + s.planes;
        ga.wq = static_cast<const uint32_t *>(wt_packed);
        ga.rows = p.rows;
        ga.index = lora->index;
        ga.hid = sa.out;
        ga.down = sa.down;
        ga.low = lora->a;
        ga.y = dx;
        ga.m = (int)m;
        ga.hw = hw;
        ga.K = cout;
        ga.KW = (cout + 15) / 16;
        ga.Nc = cin;
        ga.rank = lora->rank;
        ga.adapters = lora->adapters;
        ga.planes = planes;
        ga.Kp = sa.Kp;
        lora_gemm(ga, lora->type, dy_type, true, st);
    }
    if (da || db) {
        LoraGradBoth all{};
        if (da) all.a = {x, sa.out_step, nullptr, reinterpret_cast<float *>(ws + s.part_a), da, cin, (cin + 511) / 512};
        if (db) all.b = {dy, hid, lora->scale, reinterpret_cast<float *>(ws + s.part_b), db, cout, (cout + 511) / 512};
        all.rows = p.rows;
        all.chunks = p.chunks;
        all.groups = p.groups;
        all.rank = lora->rank;
        all.adapters = lora->adapters;
        all.chunk = kLoraChunk;
        by_real_type(dy_type, [&](auto t) {
            const unsigned cols = (unsigned)(all.a.blocks + all.b.blocks);
            if (lora->rank <= 16)
                hipLaunchKernelGGL((lora_grad_kernel<decltype(t), 1>), dim3((unsigned)s.nchunks, cols, 1), dim3(256), 0, st, all);
            else
                hipLaunchKernelGGL((lora_grad_kernel<decltype(t), 2>), dim3((unsigned)s.nchunks, cols, (unsigned)((lora->rank + 31) / 32)), dim3(256), 0, st, all);
        });
        hipLaunchKernelGGL(lora_grad_sum_kernel, dim3((unsigned)(lora->adapters * lora->rank), (unsigned)((da ? (cin + 1023) / 1024 : 0) + (db ? (cout + 1023) / 1024 : 0))),
                           dim3(256), 0, st, all);
    }
    return check_launch();
}
