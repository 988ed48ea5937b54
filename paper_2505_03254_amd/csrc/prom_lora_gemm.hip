// y = (rows x ternary weights) scaled, plus the rows' low-rank terms: the product behind prom_pw_conv_lora and, on 16-bit planes,
// the gradient of its activations.
//
// Tiled kernel.  As in the kernel of wide layers (prom_pw_gemm.hip) the k loop is outermost over a workgroup's tile, a wavefront owns
// 16*PT rows x 64 channels, decodes its own packed codes in registers and reads the rows' operands from two LDS slabs, filled a
// step ahead.  A step is 128 bytes of every row: 128 int8 or 64 bf16, two matrix instructions deep per accumulator, so
// that a barrier stands against 2*4*PT of them.
// A code is two's complement in two bits.  At the top of a byte it reads as 0, 64 or -64; at the top of 16 bits as the bf16 or f16 0, 2 or
// -2: decoding is a shift and a mask, 7 instructions for 16 codes in int8 and 15 in bf16.  The sums are 64 (exact in int32)
// and 2 times too large; the first is shifted back, the second has its half in the input planes.
// Rows are taken in the order of their adapters, so a wavefront's rows hold few of them: per adapter it loads its channels'
// factors once and adds hid b with the accumulators as the third operand.  hid goes in as bf16 planes side by side: of
// the 32 deep instruction 16 ranks take the first plane and 16 the second; a second instruction carries the third plane
// and the factors' second one where the types have them, a third one the product of both second planes.
// 8192 x 4096 -> 4096: int8 118 us at rank 16 (2.3 Pop/s; the library's plain int8 product reaches 2.2 on this card), one plane 207 to 241
// (1.14 to 1.33 PF/s; 1.43).  Matrix cores are busy for 39 % (rank 32) and 48 % of the nominal clock's cycles; the rest is the ends of a tile (every 16 ranks 3 to 4 us a round of
// tiles) and the waits of the two wavefronts of a SIMD for LDS and each other.  Small tiles are chains of latencies: a step takes 0.4 to 0.5 us however little it
// multiplies.
#include "prom_lora_gemm.h"
#include "prom_device.h"
#include "prom_launch.h"
#include "prom_pw_stream.h"

namespace prom {

// 16 codes of a word as 64 times their values, in the order of decode_word
__device__ __forceinline__ v4i decode_word_64(uint32_t w)
{
    return v4i{(int)((w << 6) & 0xc0c0c0c0u), (int)((w << 4) & 0xc0c0c0c0u), (int)((w << 2) & 0xc0c0c0c0u), (int)(w & 0xc0c0c0c0u)};
}
// 8 codes (H: first or second 8 of the 16) as bf16 (the same bits as f16) of twice their values, channels in the order 0, 2, 1, 3 of every four
template <int H> __device__ __forceinline__ v8bf decode_half_bf16(uint32_t w)
{
    constexpr int d = 2 * H;
    const v4i r = {(int)((w << (14 - 2 * d)) & 0xc000c000u), (int)((H ? w << 2 : w << 6) & 0xc000c000u),
                   (int)((w << (12 - 2 * d)) & 0xc000c000u), (int)((H ? w : w << 4) & 0xc000c000u)};
    return __builtin_bit_cast(v8bf, r);
}

// (acc * w_scale) * x_step + bias in three float32 operations, as prom_pw_conv_dynq forms it; acc64 is 64 times the sum
__device__ __forceinline__ float base_value(int acc64, float w_scale, float x_step, float bias)
{
    return add_f32(mul_f32(mul_f32((float)(acc64 >> 6), w_scale), x_step), bias);
}

template <typename TO, typename TA> struct LowPlanes {
    // one instruction for bf16 factors and 16-bit results (f16 tells 11 bits apart: hid in 16 are enough); two otherwise
    static constexpr int HID = sizeof(TO) == 4 ? 3 : 2;
    static constexpr int LOW = planes_of<TA>();
    static constexpr bool SECOND = HID == 3 || LOW == 2;
    static constexpr bool THIRD = HID == 3 && LOW == 2;  // the second planes of both
};

constexpr int kNone = 0x7fffffff;  // the adapter of rows without one
constexpr int kCodeStep = 64 * 16 + 32;  // a wavefront's words of a word step: [64 channels][4 words]
constexpr int kCodeBytes = 4 * kCodeStep;

template <int PT, int NW, int KG> struct LoraGeom {
    static constexpr int NT = 64 * NW;                      // threads of a group
    static constexpr int TM = 16 * PT;
    static constexpr int TN = 64 * NW;
    static constexpr int NQ = TM * 8 / NT;  // 16-byte pieces of a step per thread
    static constexpr int SLAB = TM * 128;
    static constexpr int OUT = 16 * (64 * 4 + 16);  // a wavefront's 16 rows x 64 channels on their way out (float32 at most)
    static constexpr int WAVE = kCodeBytes > OUT ? kCodeBytes : OUT;
    static constexpr int LOWS = 16 * (TN * 2 + 16);  // factors of 16 ranks
    static_assert(2 * LOWS <= NW * WAVE, "two buffers of them fit the wavefronts' own places");
    // steps of rows requested ahead in registers: a step of the large tile is 64 instructions of 16 cycles for each of two wavefronts, long
    // enough for one; with smaller tiles a step ends long before the next one's loads arrive (32 x 128, 52 steps: 34 us with one)
    static constexpr int D = PT == 8 ? 1 : PT == 4 ? 2 : 4;
    static constexpr int GROUP = 2 * SLAB + NW * WAVE;      // LDS of a group: slabs, then the wavefronts' own places
    static_assert(KG == 1 || PT * 4 * 1024 * NW <= GROUP, "a group's sums fit its place");
    static constexpr int ROWS = KG * GROUP;                 // row, adapter, step of every row
    static constexpr int CHANS = ROWS + TM * 12;            // w_scale, bias of every channel
    static constexpr size_t LDS = (size_t)CHANS + TN * 8;
};

// PLANES: planes instead of int8 (aligned and padded by their writer).
// KG groups of NW wavefronts share the steps of a tile, each with slabs and codes of its own; their sums meet in LDS, and the first group goes on.
template <int PT, int NW, int KG, bool PLANES, typename TO, typename TA>
__global__ __launch_bounds__(64 * NW * KG, 2) void lora_gemm_kernel(const LoraGemmArgs a, int ntiles)
{
    using G = LoraGeom<PT, NW, KG>;
    constexpr int NQ = G::NQ;
    using Acc = typename std::conditional<PLANES, v4f, v4i>::type;
    constexpr bool SCALED = PLANES && kScaledPlane<TO>;  // one f16 plane, a factor per row
    extern __shared__ __align__(16) unsigned char all_lds[];
    const int tid = threadIdx.x % G::NT;  // in the group
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / G::NT);
    unsigned char *lds = all_lds + kg * G::GROUP;
    const int j = lane & 15, g = lane >> 4;
    const int lid = logical_block_id();
    const int mtiles = (a.m + G::TM - 1) / G::TM;
    const int ntile = lid % ntiles, mtile = lid / ntiles;
    if (mtile >= mtiles) return;
    const int n0 = ntile * G::TN + 64 * wave;  // this wavefront's first channel
    const int m0 = mtile * G::TM;
    const int K = a.K, KW = a.KW, Nc = a.Nc;

    // ---- rows: piece idx = tid + NT*q of a slab is slot idx & 7 of row idx >> 3 and holds the row's piece slot ^ ((row >> 1) & 7): two rows
    // fill LDS's 64 banks, so that 16 rows' operands lie in different ones
    const int row_bytes = PLANES ? a.planes * a.Kp * 2 : K;
    const int piece = (tid & 7) ^ ((tid >> 4) & 7);
    const unsigned char *src[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int pos = min(m0 + ((tid + G::NT * q) >> 3), a.m - 1);
        const int row = PLANES ? pos : a.rows[pos];
        src[q] = static_cast<const unsigned char *>(a.x) + (size_t)row * row_bytes;
    }
    // Steps in the order they are taken: what is left behind the whole ones comes first, read piece by piece with zeros behind the row's
    // end, so that everything later loads whole pieces without a test (the order of a sum of integers is free; planes are padded).
    const int whole = row_bytes >> 7;
    const int first = !PLANES && (row_bytes & 127) ? 1 : 0;
    const int steps = whole + first;
    // the group's turn i is step KG*i + kg; every group makes the same number of turns (they share the barriers), the last of them with zeros
    // where there is no step left
    const int turns = (steps + KG - 1) / KG;
    constexpr int D = G::D;
    v4i xring[D][NQ];  // turn i in slot i % D
    // (what is asked for behind the last step repeats it, and a row without a whole step reads the row numbers: neither is used.  A
    // test around the loads would make the compiler wait for the newest instead of the one it needs)
    auto load_x = [&](int i_, v4i(&xr)[NQ]) __attribute__((always_inline)) {
        const int at = 128 * max(min(KG * i_ + kg, steps - 1) - first, 0) + 16 * piece;
#pragma unroll
        for (int i = 0; i < NQ; ++i) xr[i] = *reinterpret_cast<const v4i_u *>(src[i] + at);
    };
    auto put_x = [&](int i_, int slab, const v4i(&xr)[NQ]) __attribute__((always_inline)) {
        const bool none = KG > 1 && KG * i_ + kg >= steps;
#pragma unroll
        for (int q = 0; q < NQ; ++q) *reinterpret_cast<v4i *>(lds + slab * G::SLAB + (tid + G::NT * q) * 16) = none ? v4i{0, 0, 0, 0} : xr[q];
    };

    // ---- codes: 16 words of each of the wavefront's 64 channels at a time, 4 word steps; instruction r of a load: channel
    // 16*r + (lane >> 2), word step lane & 3.  A word step is 64 channels of input; planes follow each other.  Words past a row's end are replaced
    // by its last one: they meet zeros of the other operand.
    constexpr int WS = PLANES ? 1 : 2;   // word steps of a step
    constexpr int GS = 4 / WS;           // turns of a set of codes
    unsigned char *codes = lds + 2 * G::SLAB + wave * G::WAVE;
    const int wsteps = PLANES ? a.Kp >> 6 : 0x7fffffff;  // word steps of one plane
    const int wpiece = lane & 3;
    const uint32_t *wrow[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) wrow[r] = a.wq + (size_t)min(n0 + 16 * r + (lane >> 2), Nc - 1) * KW;
    // sets of codes requested ahead: with small tiles one of int8 lasts two short steps, and codes come from memory as late as rows do
    constexpr int DW = D > 1 && !PLANES ? 2 : 1;
    struct Words {
        v4i v[4];
        int shift;  // words that lie before the ones wanted: a row's last ones are read as the row's last four
    } wring[DW];    // set q in slot q % DW
    auto load_w = [&](int set, Words &w) __attribute__((always_inline)) {
        const int q = min(KG * (GS * set + wpiece / WS) + kg, steps - 1);
        int ws = WS * (q < first ? whole : q - first) + wpiece % WS;
        if constexpr (PLANES) {
            if (ws >= wsteps) ws -= wsteps;
            if (ws >= wsteps) ws -= wsteps;
        }
        const int from = max(min(4 * ws, KW - 4), 0);
        w.shift = min(4 * ws - from, 3);
#pragma unroll
        for (int r = 0; r < 4; ++r) w.v[r] = *reinterpret_cast<const v4i_u *>(wrow[r] + from);
    };
    unsigned char *wput = codes + wpiece * kCodeStep + (lane >> 2) * 16;
    const unsigned char *wget = codes + j * 16 + g * 4;
    auto put_w = [&](const Words &w) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v4i v = w.v[r];
            if ((KW & 3) != 0) {
                const bool odd = w.shift & 1, two = w.shift & 2;
                const int x0 = odd ? v[1] : v[0], x1 = odd ? v[2] : v[1], x2 = odd ? v[3] : v[2];
                v = v4i{two ? x2 : x0, two ? v[3] : x1, x2, v[3]};
            }
            *reinterpret_cast<v4i *>(wput + 256 * r) = v;
        }
    };

    Acc acc[PT][4];
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[i][t] = Acc{0, 0, 0, 0};

    int *lrow = reinterpret_cast<int *>(all_lds + G::ROWS);  // [TM] row, [TM] adapter (kNone: none), [TM] step
    float *lstep = reinterpret_cast<float *>(lrow + 2 * G::TM);
    float *lws = reinterpret_cast<float *>(all_lds + G::CHANS);  // [TN] w_scale, [TN] bias
    if (KW >= 4) load_w(0, wring[0]);
    else {  // one group holds every word of such a row; nothing behind it is used, and it is read from where there is something
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int e = 0; e < 4; ++e) wring[0].v[r][e] = (int)wrow[r][min(e, KW - 1)];
            wrow[r] = reinterpret_cast<const uint32_t *>(a.rows);
        }
        wring[0].shift = 0;
    }
    if constexpr (DW == 2) load_w(1, wring[1]);
    // What the epilogue needs first: a row's number, adapter and step by the thread that will bring its hid in (half tid & 1 of 16 ranks of
    // row tid >> 1), a channel's scale and bias, and the first ranks of hid and of the first adapter's factors.  With small tiles the whole
    // product takes no longer than these dependent loads, so they leave now and stay in registers; the large tile has none to spare.
    constexpr bool EARLY = PT < 8;
    constexpr int LP = G::TN * 2 + 16;  // bytes between ranks
    const TA *low = static_cast<const TA *>(a.low);
    Piece<TA, 8> lv[2];
    auto load_low = [&](int l, int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int idx = tid + G::NT * q;
            const int r = idx / (G::TN / 8), c = ntile * G::TN + idx % (G::TN / 8) * 8;
            lv[q].load_some(low + ((size_t)l * a.rank + min(r0 + r, a.rank - 1)) * Nc + c, r0 + r < a.rank ? Nc - c : 0);
        }
    };
    auto element = [&](int row) __attribute__((always_inline)) { return a.hw == 1 ? row : row / a.hw; };
    const int hrow = tid >> 1, hhalf = tid & 1;
    int my_row = a.rows[min(m0 + min(hrow, G::TM - 1), a.m - 1)];
    int my_adapter = a.index[element(my_row)];
    if (hrow >= G::TM || m0 + hrow >= a.m || my_adapter < 0 || my_adapter >= a.adapters) my_adapter = kNone;
    int adapter0 = a.index[element(a.rows[m0])];  // the smallest one of the tile: its rows are sorted
    if (adapter0 < 0 || adapter0 >= a.adapters) adapter0 = kNone;
    float my_step = 0.0f, my_ws = 0.0f, my_bias = 0.0f, hscale = 1.0f;
    if constexpr (!PLANES) {
        const int c = min(ntile * G::TN + tid, Nc - 1);
        my_step = a.step[element(my_row)];
        my_ws = a.w_scale[c];
        if (a.bias) my_bias = a.bias[c];
    }
    if constexpr (SCALED) my_step = a.down[my_row];
    auto put_info = [&]() __attribute__((always_inline)) {
        if (hhalf == 0 && hrow < G::TM) {
            lrow[hrow] = my_row;
            lrow[G::TM + hrow] = my_adapter;
            lstep[hrow] = my_step;
        }
        if constexpr (!PLANES) {
            lws[tid] = my_ws;
            lws[G::TN + tid] = my_bias;
        }
    };
    Piece<float, 8> hv;
    const float *hfrom = a.hid;
    auto load_hid = [&](int r0) __attribute__((always_inline)) { hv.load_some(hfrom + r0, my_adapter != kNone ? a.rank - r0 - 8 * hhalf : 0); };
    auto load_first = [&]() __attribute__((always_inline)) {
        hfrom = a.hid + (size_t)my_row * a.rank + 8 * hhalf;
        if (adapter0 == kNone) return;
        load_hid(0);
        if (a.scale && my_adapter != kNone) hscale = a.scale[my_adapter];
        load_low(adapter0, 0);
    };
    if constexpr (!EARLY) put_info();
    if (first && kg == 0) {
        const int at = 128 * whole + 16 * piece;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            Piece<int8_t, 16> v;
            v.load_some(reinterpret_cast<const int8_t *>(src[q] + at), row_bytes - at);
            xring[0][q] = __builtin_bit_cast(v4i, v);
        }
    }
    if (whole == 0)
#pragma unroll
        for (int q = 0; q < NQ; ++q) src[q] = reinterpret_cast<const unsigned char *>(a.rows);
    if (!(first && kg == 0)) load_x(0, xring[0]);
#pragma unroll
    for (int d = 1; d < D; ++d) load_x(d, xring[d]);
    put_w(wring[0]);
    load_w(DW, wring[0]);
    put_x(0, 0, xring[0]);
    load_x(D, xring[0]);
    if constexpr (EARLY)
        if (kg == 0) load_first();
    lds_only_barrier();

    const int sw = (j >> 1) & 7;
    auto step = [&](auto turn, int s) __attribute__((always_inline)) {  // the group's turn s; turn = s % 4
        const int TURN = turn, NEXT = (TURN + 1) % D;
        const unsigned char *slab = lds + (TURN & 1) * G::SLAB + j * 128;
        uint32_t wc[WS][4];
#pragma unroll
        for (int h = 0; h < WS; ++h)
#pragma unroll
            for (int t = 0; t < 4; ++t) wc[h][t] = *reinterpret_cast<const uint32_t *>(wget + (WS * (TURN % GS) + h) * kCodeStep + 256 * t);
        put_x(s + 1, (TURN + 1) & 1, xring[NEXT]);
        load_x(s + 1 + D, xring[NEXT]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4i B[PT];
            const int p = PLANES ? 2 * g + h : 4 * h + g;
#pragma unroll
            for (int i = 0; i < PT; ++i) B[i] = *reinterpret_cast<const v4i *>(slab + i * 2048 + ((p ^ sw) << 4));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if constexpr (PLANES) {
                    const v8bf A = h ? decode_half_bf16<1>(wc[0][t]) : decode_half_bf16<0>(wc[0][t]);
#pragma unroll
                    for (int i = 0; i < PT; ++i) {
                        if constexpr (SCALED) acc[i][t] = mfma_f16(__builtin_bit_cast(v8h, A), __builtin_bit_cast(v8h, B[i]), acc[i][t]);
                        else acc[i][t] = mfma_bf16(A, __builtin_bit_cast(v8bf, B[i]), acc[i][t]);
                    }
                } else {
                    const v4i A = decode_word_64(wc[h][t]);
#pragma unroll
                    for (int i = 0; i < PT; ++i) acc[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, B[i], acc[i][t], 0, 0, 0);
                }
            }
        }
        if (TURN % GS == GS - 1) {  // (LDS operations of a wavefront keep their order, and no other one reads these words)
            Words &w = wring[(TURN / GS + 1) % DW];
            put_w(w);
            load_w(s / GS + 1 + DW, w);
        }
        lds_only_barrier();
    };
    static_assert(4 % D == 0 && 4 % GS == 0, "the turns below");
    int s = 0;
    if constexpr (D == 1) {  // (the large tile's registers do not hold four turns' code: 142 us against 182)
        for (; s < turns; ++s) step(s & 3, s);
    } else {
        for (; s + 4 <= turns; s += 4) {
            step(std::integral_constant<int, 0>{}, s);
            step(std::integral_constant<int, 1>{}, s + 1);
            step(std::integral_constant<int, 2>{}, s + 2);
            step(std::integral_constant<int, 3>{}, s + 3);
        }
        if (s < turns) step(std::integral_constant<int, 0>{}, s);
        if (s + 1 < turns) step(std::integral_constant<int, 1>{}, s + 1);
        if (s + 2 < turns) step(std::integral_constant<int, 2>{}, s + 2);
    }

    if constexpr (KG > 1) {
        if (kg > 0) {
#pragma unroll
            for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int t = 0; t < 4; ++t) *reinterpret_cast<Acc *>(lds + ((wave * PT + i) * 4 + t) * 1024 + lane * 16) = acc[i][t];
        }
        lds_only_barrier();
        if (kg > 0) return;  // (a barrier waits for the wavefronts that are left)
#pragma unroll
        for (int o = 1; o < KG; ++o)
#pragma unroll
            for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[i][t] += *reinterpret_cast<const Acc *>(all_lds + o * G::GROUP + ((wave * PT + i) * 4 + t) * 1024 + lane * 16);
    }

    // ---- epilogue: lane (j, g), register e of tile (i, t): row 16i + j, channel n0 + 16t + 4g + e --------------------
    // Ranks 16 at a time, adapter after adapter (the same ones in every wavefront: all own the same rows).  All threads bring the tile's hid
    // in, scaled and split into planes, one half of 8 ranks of a row each, into the slabs that are free by now, and an adapter's
    // factors [16 ranks][TN channels] into the codes' place; both have two buffers in turn, and the next ones are on their way in
    // registers while the last ones are used.
    using L = LowPlanes<TO, TA>;
    auto put_low = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int idx = tid + G::NT * q;
            lv[q].store(reinterpret_cast<TA *>(lds + 2 * G::SLAB + buffer * G::LOWS + idx / (G::TN / 8) * LP) + idx % (G::TN / 8) * 8);
        }
    };
    if constexpr (EARLY) {
        put_info();
        lds_only_barrier();
    } else {
        my_row = lrow[min(hrow, G::TM - 1)];
        my_adapter = hrow < G::TM ? lrow[G::TM + hrow] : kNone;
        adapter0 = __builtin_amdgcn_readfirstlane(lrow[G::TM]);
        load_first();
    }
    int own[PT];  // adapter of row 16i + j
#pragma unroll
    for (int i = 0; i < PT; ++i) own[i] = lrow[G::TM + 16 * i + j];
    auto next_adapter = [&](int after) __attribute__((always_inline)) {  // the wavefront's smallest one above `after`
        int next = kNone;
#pragma unroll
        for (int i = 0; i < PT; ++i) next = own[i] > after ? min(next, own[i]) : next;
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) next = min(next, __shfl_xor(next, o, 64));
        return __builtin_amdgcn_readfirstlane(next);
    };
    v4f z[PT][4];
    float st[PT];
    if constexpr (SCALED || !PLANES)
#pragma unroll
        for (int i = 0; i < PT; ++i) st[i] = lstep[16 * i + j];
    if constexpr (PLANES) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) z[i][t] = SCALED ? acc[i][t] * st[i] : acc[i][t];
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const v4f ws = *reinterpret_cast<const v4f *>(lws + 64 * wave + 16 * t + 4 * g);
            const v4f bi = *reinterpret_cast<const v4f *>(lws + G::TN + 64 * wave + 16 * t + 4 * g);
#pragma unroll
            for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i][t][e] = base_value(acc[i][t][e], ws[e], st[i], bi[e]);
        }
    }
    if (adapter0 != kNone) {
        for (int r0 = 0, turn = 0, buffer = 0; r0 < a.rank; r0 += 16, turn ^= 1) {
            unsigned char *planes = lds + turn * G::SLAB;  // [TM][4 slots of 16 bytes], twice
            if (hrow < G::TM) {
                v8bf s0, s1, s2;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t s[3];
                    split<3>(hv.e[e] * hscale, s);
                    s0[e] = s[0];
                    s1[e] = s[1];
                    s2[e] = s[2];
                }
                unsigned char *to = planes + hrow * 64;
                const int x = (hrow >> 1) & 3;
                *reinterpret_cast<v8bf *>(to + ((hhalf ^ x) << 4)) = s0;
                *reinterpret_cast<v8bf *>(to + (((2 + hhalf) ^ x) << 4)) = s1;
                if constexpr (L::SECOND) {
                    *reinterpret_cast<v8bf *>(to + G::TM * 64 + ((hhalf ^ x) << 4)) = s0;
                    *reinterpret_cast<v8bf *>(to + G::TM * 64 + (((2 + hhalf) ^ x) << 4)) = s2;
                }
            }
            for (int l = adapter0; l != kNone;) {
                put_low(buffer);
                lds_only_barrier();
                const int after = next_adapter(l);
                if (after != kNone) load_low(after, r0);
                else if (r0 + 16 < a.rank) {
                    load_low(adapter0, r0 + 16);
                    load_hid(r0 + 16);
                }
                v8bf A1[4], A2[L::SECOND ? 4 : 1], A3[L::THIRD ? 4 : 1];
                const TA *factors = reinterpret_cast<const TA *>(lds + 2 * G::SLAB + buffer * G::LOWS + 8 * (g & 1) * LP) + 64 * wave + j;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        bf16_t s[L::LOW];
                        const TA v = factors[e * (LP / 2) + 16 * t];
                        if constexpr (std::is_same<TA, bf16_t>::value) s[0] = v;
                        else split<L::LOW>((float)v, s);
                        A1[t][e] = s[0];
                        if constexpr (L::SECOND) A2[t][e] = g < 2 ? (L::LOW == 2 ? s[L::LOW - 1] : (bf16_t)0.0f) : s[0];
                        if constexpr (L::THIRD) A3[t][e] = g < 2 ? (bf16_t)0.0f : s[L::LOW - 1];
                    }
#pragma unroll
                for (int i = 0; i < PT; ++i) {
                    const bool mine = own[i] == l;
                    const unsigned long long here = __ballot(mine);
                    if (here == 0) continue;
                    const unsigned char *from = planes + (16 * i + j) * 64 + ((g ^ ((j >> 1) & 3)) << 4);
                    const v8bf b1 = *reinterpret_cast<const v8bf *>(from);
                    v8bf b2;
                    if constexpr (L::SECOND) b2 = *reinterpret_cast<const v8bf *>(from + G::TM * 64);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        v4f v = mfma_bf16(A1[t], b1, z[i][t]);
                        if constexpr (L::SECOND) v = mfma_bf16(A2[t], b2, v);
                        if constexpr (L::THIRD) v = mfma_bf16(A3[t], b1, v);
                        if (here == ~0ull) z[i][t] = v;
                        else  // (what another adapter makes of this row's hid is dropped, whatever it is)
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[i][t][e] = mine ? v[e] : z[i][t][e];
                    }
                }
                l = after;
                buffer ^= 1;
            }
        }
        lds_only_barrier();
    }
    // out through the wavefront's own LDS: 16 rows x 64 channels at a time, rows in whole runs
    constexpr int PITCH = 64 * (int)sizeof(TO) + 16;
    constexpr int VE = 16 / sizeof(TO), PR = 64 / VE;  // elements of a piece, pieces of a row
    TO *y = static_cast<TO *>(a.y);
#pragma unroll
    for (int i = 0; i < PT; ++i) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            Piece<TO, 4> o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o.e[e] = (TO)z[i][t][e];
            o.store(reinterpret_cast<TO *>(codes + j * PITCH) + 16 * t + 4 * g);
        }
#pragma unroll
        for (int q = 0; q < 16 * PR / 64; ++q) {
            const int idx = lane + 64 * q;
            const int rr = idx / PR, c = idx % PR * VE;
            Piece<TO, VE> o;
            o.load(reinterpret_cast<const TO *>(codes + rr * PITCH) + c);
            if (m0 + 16 * i + rr < a.m) o.store_some(y + (size_t)lrow[16 * i + rr] * Nc + n0 + c, Nc - n0 - c);
        }
    }
}

// ---- a few rows -----------------------------------------------------------------------------------------------
// Up to 64 rows: a workgroup owns 16 CT channels and 16 MT rows, its 8 wavefronts share the input channels 256 at a time, the sums meet in LDS.
// Four lanes read 64 bytes of a row (and 16 of a channel's codes) in one instruction: every row passes the texture addresser
// in whole runs.  The low-rank term is one dot product over the ranks per output on the vector ALU, every row with its own adapter; its
// operands are requested before the product, which they do not depend on.  Bound by latency, then by the adapters' bytes.
// FUSE: for a token or two every workgroup forms hid itself (rank * cin * 2 bytes a row out of L2, 131 KB at 4096 channels and rank 16, while
// the product's own loads are on their way) and no launch goes before this one: 10.2 us for 1 token of 4096 -> 4096 against 3.2 + 5.6 in two
// launches, which cost the host 2 us more.  64 tokens with 64 adapters: 12.3 us.
template <typename TO, typename TA, int MT, int CT, bool FUSE>
__global__ __launch_bounds__(512) void lora_gemm_few_kernel(const LoraGemmArgs a)
{
    __shared__ v4i red[8][CT * MT][64];
    __shared__ float formed[FUSE ? kFuseMost : 1];
    constexpr int RP = 16;  // ranks requested ahead
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, g = lane >> 4;
    const int row_blocks = (a.m + 16 * MT - 1) / (16 * MT);  // (workgroups of the same channels are neighbours)
    const int lid = logical_block_id();
    const int n0 = lid / row_blocks * 16 * CT, m0 = lid % row_blocks * 16 * MT;
    if (n0 >= a.Nc) return;
    const int K = a.K, KW = a.KW;

    // what the thread will write: two channels of a row
    const int mine = tid / (8 * CT), cc = 2 * (tid % (8 * CT)), c = n0 + cc;
    const bool out = mine < 16 * MT && m0 + mine < a.m && c < a.Nc;
    const int row = min(m0 + mine, a.m - 1), channels = out ? a.Nc - c : 0;
    const int el = a.hw == 1 ? row : row / a.hw;
    const int l = a.index[el];
    const bool has = out && l >= 0 && l < a.adapters;
    const float st = a.step[el];
    const TA *low = static_cast<const TA *>(a.low) + (size_t)(has ? l : 0) * a.rank * a.Nc + c;
    const float *hid = a.hid + (size_t)row * a.rank;
    Piece<TA, 2> b[RP];
    float h[RP];
    float f = 0.0f;
    const uint32_t *wrow[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) wrow[t] = a.wq + (size_t)min(n0 + 16 * t + j, a.Nc - 1) * KW;
    const int8_t *xrow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xrow[i] = static_cast<const int8_t *>(a.x) + (size_t)min(m0 + 16 * i + j, a.m - 1) * K;
    v4i acc[CT][MT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[t][i] = v4i{0, 0, 0, 0};
    // N steps' loads leave before the first is used; `then` is called between the two
    auto steps = [&](auto whole, auto count, int k, auto then) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int N = decltype(count)::value;
        uint32_t w[N][CT][4];
        Piece<int8_t, 16> v[N][MT][4];
#pragma unroll
        for (int s = 0; s < N; ++s)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int k0 = k + 2048 * s + 64 * q + 16 * g;
#pragma unroll
                for (int t = 0; t < CT; ++t) w[s][t][q] = wrow[t][WHOLE ? k0 >> 4 : min(k0 >> 4, KW - 1)];  // (past the row's end it meets zeros)
#pragma unroll
                for (int i = 0; i < MT; ++i) v[s][i][q].load_some(xrow[i] + k0, WHOLE ? 16 : K - k0);
            }
        then();
#pragma unroll
        for (int s = 0; s < N; ++s)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const v4i A = decode_word_64(w[s][t][q]);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        acc[t][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, __builtin_bit_cast(v4i, v[s][i][q]), acc[t][i], 0, 0, 0);
                }
            }
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    Piece<float, 2> ws, bi;
    auto adapters = [&]() __attribute__((always_inline)) {
        ws.load_some(a.w_scale + c, channels);
        bi.load_some(a.bias + c, a.bias ? channels : 0);
        if (has) {
            f = a.scale[l];
#pragma unroll
            for (int r = 0; r < RP; ++r) {
                const int rr = min(r, a.rank - 1);
                b[r].load_some(low + (size_t)rr * a.Nc, channels);
                if constexpr (!FUSE) h[r] = hid[rr];
            }
        }
        if constexpr (FUSE) {
            for (int p = wave; p < a.m * a.rank; p += 8) {  // a wavefront per row and rank
                const int prow = p / a.rank, r = p - prow * a.rank;
                const int pel = a.hw == 1 ? prow : prow / a.hw;
                const int pl = a.index[pel];
                float s = 0.0f;
                if (pl >= 0 && pl < a.adapters) {
                    const int8_t *x = static_cast<const int8_t *>(a.x) + (size_t)prow * K;
                    const TA *w = static_cast<const TA *>(a.first) + ((size_t)pl * a.rank + r) * K;
                    auto dot = [&](auto whole, int k, int u) __attribute__((always_inline)) {
                        constexpr bool WHOLE = decltype(whole)::value;
                        constexpr int N = WHOLE ? 8 : 1;
                        Piece<int8_t, 8> xv[N];
                        Piece<TA, 8> wv[N];
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            const int k0 = k + 512 * (n < u ? n : 0) + 8 * lane;
                            xv[n].load_some(x + k0, WHOLE ? 8 : K - k0);
                            wv[n].load_some(w + k0, WHOLE ? 8 : K - k0);
                        }
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            if (n >= u) break;
#pragma unroll
                            for (int e = 0; e < 8; ++e) s += (float)xv[n].e[e] * (float)wv[n].e[e];
                        }
                    };
                    const int kw = K & ~511;
                    for (int k = 0; k < kw; k += 4096) dot(std::true_type{}, k, min(8, (kw - k) >> 9));
                    if (kw < K) dot(std::false_type{}, kw, 1);
                    s = wave_sum_f32(s) * a.step[pel];
                }
                if (lane == 0) {
                    formed[p] = s;
                    if (lid == 0) a.hid_out[p] = s;
                }
            }
        }
    };
    auto nothing = [] {};
    const int end = K & ~255;
    int k = 256 * wave;
    if (k + 2048 < end) {
        steps(std::true_type{}, Two{}, k, adapters);
        k += 4096;
    } else if (k < end) {
        steps(std::true_type{}, One{}, k, adapters);
        k += 2048;
    } else
        adapters();
    for (; k < end; k += 2048) steps(std::true_type{}, One{}, k, nothing);
    if (end < K && (end >> 8 & 7) == wave) steps(std::false_type{}, One{}, end, nothing);
#pragma unroll
    for (int i = 0; i < CT * MT; ++i) red[wave][i][lane] = acc[i / MT][i % MT];
    __syncthreads();
    if (!out) return;
    int s0 = 0, s1 = 0;
    {
        const int from = (mine & 15) + 16 * (cc >> 2 & 3), e = cc & 3, at = (cc >> 4) * MT + (mine >> 4);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const int *p = reinterpret_cast<const int *>(&red[w][at][from]) + e;
            s0 += p[0];
            s1 += p[1];
        }
    }
    float z0 = base_value(s0, ws.e[0], st, bi.e[0]), z1 = base_value(s1, ws.e[1], st, bi.e[1]);
    if (has) {
        float l0 = 0.0f, l1 = 0.0f;
        if constexpr (FUSE) hid = formed + row * a.rank;
#pragma unroll
        for (int r = 0; r < RP; ++r) {
            if constexpr (FUSE) h[r] = hid[min(r, a.rank - 1)];
            const float v = r < a.rank ? h[r] : 0.0f;
            l0 += r < a.rank ? v * (float)b[r].e[0] : 0.0f;
            l1 += r < a.rank ? v * (float)b[r].e[1] : 0.0f;
        }
#pragma unroll 16
        for (int r = RP; r < a.rank; ++r) {
            Piece<TA, 2> v;
            v.load_some(low + (size_t)r * a.Nc, channels);
            l0 += hid[r] * (float)v.e[0];
            l1 += hid[r] * (float)v.e[1];
        }
        z0 += f * l0;
        z1 += f * l1;
    }
    Piece<TO, 2> o;
    o.e[0] = (TO)z0;
    o.e[1] = (TO)z1;
    o.store_some(static_cast<TO *>(a.y) + (size_t)row * a.Nc + c, channels);
}

// ---- launch ----------------------------------------------------------------------------------------------------
template <int PT, int NW, int KG, bool PLANES, typename TO, typename TA> static void gemm_launch(const LoraGemmArgs &a, hipStream_t st)
{
    using G = LoraGeom<PT, NW, KG>;
    const int ntiles = (a.Nc + G::TN - 1) / G::TN;
    const long long mtiles = (a.m + G::TM - 1) / G::TM;
    static_assert(G::LDS <= 64 * 1024, "what a launch takes without asking");
    hipLaunchKernelGGL((lora_gemm_kernel<PT, NW, KG, PLANES, TO, TA>), dim3((unsigned)((mtiles * ntiles + 7) / 8 * 8)), dim3(G::NT * KG), G::LDS, st, a, ntiles);
}

template <bool PLANES, typename TO, typename TA> static void gemm_pick(const LoraGemmArgs &a, hipStream_t st)
{
    // The largest tile that still gives every compute unit a workgroup (the largest of all two: it runs two at a time), and with few small
    // tiles two groups of wavefronts that halve the chain of steps.  Measured (us, tiles 128x256 / 64x256 / 32x256 / 32x128 / 32x128 by two
    // groups, int8): 8192 x 4096 x 4096 118 / 130 / 186 / 191 / 232, 2048 x 4096 x 4096 47 / 39 / 52 / 53 / 64,
    // 512 x 4096 x 4096 39 / 25 / 21 / 24 / 20, 128 x 4096 x 4096 45 / 27 / 21 / 18 / 14, 12544 x 960 x 160 23 / 16 / 15 / 15 / 22; three planes of
    // 1671 x 2474 x 457 - / 72 / 56 / 51 / 34 (by three groups 32); 100 x 500 x 600, 8 steps, - / 14 / 12 / 12 / 10.
    auto tiles = [&](int tm, int tn) { return (long long)((a.m + tm - 1) / tm) * ((a.Nc + tn - 1) / tn); };
    const int steps = PLANES ? a.planes * a.Kp / 64 : (a.K + 127) / 128;
    if (tiles(32, 128) <= 512 && steps >= 8) gemm_launch<2, 2, 2, PLANES, TO, TA>(a, st);
    else if (a.Nc <= 128) gemm_launch<2, 2, 1, PLANES, TO, TA>(a, st);  // half of a wider tile would be empty
    else if (tiles(128, 256) >= 512) gemm_launch<8, 4, 1, PLANES, TO, TA>(a, st);
    else if (tiles(64, 256) >= 256) gemm_launch<4, 4, 1, PLANES, TO, TA>(a, st);
    else if (tiles(32, 256) >= 256) gemm_launch<2, 4, 1, PLANES, TO, TA>(a, st);
    else gemm_launch<2, 2, 1, PLANES, TO, TA>(a, st);
}

template <typename F> static void by_types(int adapter_type, int out_type, F f)
{
    if (adapter_type == PROM_BF16) {
        if (out_type == PROM_F32) f(float{}, bf16_t{});
        else f(bf16_t{}, bf16_t{});
    } else {
        if (out_type == PROM_F32) f(float{}, f16_t{});
        else f(f16_t{}, f16_t{});
    }
}

void lora_gemm(const LoraGemmArgs &a, int adapter_type, int out_type, bool planes, hipStream_t st)
{
    by_types(adapter_type, out_type, [&](auto to, auto ta) {
        if (planes) gemm_pick<true, decltype(to), decltype(ta)>(a, st);
        else gemm_pick<false, decltype(to), decltype(ta)>(a, st);
    });
}

void lora_gemm_few(const LoraGemmArgs &a, int adapter_type, int out_type, hipStream_t st)
{
    by_types(adapter_type, out_type, [&](auto to, auto ta) {
        using TO = decltype(to);
        using TA = decltype(ta);
        auto go = [&](auto kernel, int rows, int channels) {
            const int blocks = ((a.Nc + channels - 1) / channels) * ((a.m + rows - 1) / rows);
            hipLaunchKernelGGL(kernel, dim3((unsigned)((blocks + 7) / 8 * 8)), dim3(512), 0, st, a);
        };
        // from 33 rows on 32 x 32 instead of all rows x 16 channels: as many workgroups, and half of the rows' bytes through each
        if (a.hid_out) go((lora_gemm_few_kernel<TO, TA, 1, 1, true>), 16, 16);  // (32 rows at most, of rank 1: two workgroups per 16 channels)
        else if (a.m <= 16) go((lora_gemm_few_kernel<TO, TA, 1, 1, false>), 16, 16);
        else if (a.m <= 32) go((lora_gemm_few_kernel<TO, TA, 2, 1, false>), 32, 16);
        else go((lora_gemm_few_kernel<TO, TA, 2, 2, false>), 32, 32);
    });
}

}  // namespace prom
