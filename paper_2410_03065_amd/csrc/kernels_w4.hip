// Products with 4-bit weights (layout: cake.h, cake_w4), and the packing of such weights.
//
// out[m][n] = sum over groups g of s[n][g] * (sum over the group's k of a[m][k] c[n][k]): the matrix cores multiply the activations by the
// codes, exact in bfloat16, a group's sum is kept apart and enters the result times its scale, one multiply-add.  Nothing is rounded
// on the way but float32 sums.  With many rows those multiply-adds cost more than the products, and the scale goes into the weight instead.
//
// Up to some 100 rows the codes' bytes bound it, then the conversion of the codes, and from 500 rows on the matrix cores.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.hpp"

namespace cake {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// v_mfma_f32_16x16x32_bf16, D[16x16] += A[16x32] * B[32x16]: lane l supplies A[l%16][8*(l/16) .. +7] and
// B[8*(l/16) .. +7][l%16], and holds D[4*(l/16) + v][l%16] in accumulator register v (0..3).
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Eight codes as bfloat16 24 + c, one shift and one three-way logic instruction a pair: a code's four bits, the upper one turned, are
// the upper bits of the fraction of 16 .. 31.  Order: elements 0 4 1 5 2 6 3 7.
__device__ __forceinline__ bf16x8 codes8(unsigned w) {
    constexpr unsigned M = 0x00780078u, B = 0x41c041c0u;
    const uint4 r = {((w << 3) & M) ^ B, ((w >> 1) & M) ^ B, ((w >> 5) & M) ^ B, ((w >> 9) & M) ^ B};
    return __builtin_bit_cast(bf16x8, r);
}
// The same order for eight activations.
__device__ __forceinline__ bf16x8 in_order(uint4 x) {
    const uint4 r = {__builtin_amdgcn_perm(x.z, x.x, 0x05040100), __builtin_amdgcn_perm(x.z, x.x, 0x07060302),
                     __builtin_amdgcn_perm(x.w, x.y, 0x05040100), __builtin_amdgcn_perm(x.w, x.y, 0x07060302)};
    return __builtin_bit_cast(bf16x8, r);
}
// The four words of the four lanes that share l % 16, transposed: word s of lane group g becomes word g of lane group s.
__device__ __forceinline__ uint4 transposed(uint4 x) {
    const auto a = __builtin_amdgcn_permlane32_swap(x.x, x.z, false, false), b = __builtin_amdgcn_permlane32_swap(x.y, x.w, false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return uint4{c[0], c[1], d[0], d[1]};
}
// The sum over LANES (4, 8 or 16) neighbouring lanes, in all of them.
template <int LANES> __device__ __forceinline__ float add_group(float y) {
    auto from = [](float v, auto ctrl) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
    y += from(y, std::integral_constant<int, 0xb1>{});                        // quad_perm 1 0 3 2
    y += from(y, std::integral_constant<int, 0x4e>{});                        // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) y += from(y, std::integral_constant<int, 0x141>{});   // row_half_mirror
    if constexpr (LANES >= 16) y += from(y, std::integral_constant<int, 0x140>{});  // row_mirror
    return y;
}
__device__ __forceinline__ unsigned word(uint4 x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

template <typename T> struct Terms { static constexpr int N = 1; };
template <> struct Terms<float> { static constexpr int N = 3; };       // 24 bits in three bfloat16
// The nearest of the finite ones: what is left of an infinity, or of a number beyond the largest, is left to the next term, and an infinity
// to the last, instead of inf - inf.  An instruction an element and term: 732 rows, 3553 outputs, 1320 inputs, groups of 32 36.3 us, without 34.4; few rows 2 % more.
__device__ __forceinline__ bf16_t finite_term(float y) {
    constexpr float MOST = 0x1.fep127f;
    return bf16_t(__builtin_amdgcn_fmed3f(y, -MOST, MOST));
}

struct Product {
    const void* a;
    const unsigned char *w, *w2;       // codes; w2: of up (SwiGLU)
    const void *s, *s2;                // scales
    void* out;
    float* parts;                      // ranges of inputs: [range][gate, up][M][N]
    int M, N, K, row_bytes, groups, epi;
};
template <typename T> __device__ __forceinline__ T silu_product(float gate, float up) { return T(gate / (1.f + expf(-gate)) * up); }

// The codes of one word, eight inputs of an output, and what a product of them with activations x is short of x times the codes themselves.
// bfloat16 activations: 24 + c in the order 0 4 1 5 2 6 3 7, and the sums of x times 24 are taken off by a product with a constant
// operand.  float32 (three terms): 16 c as they are, since the offset would cost three bits of the sums; the scale is divided by 16.
template <typename T> __device__ __forceinline__ bf16x8 operand(unsigned w) {
    if constexpr (sizeof(T) == 2) return codes8(w);
    const unsigned e = (w << 4) & 0xf0f0f0f0u, o = w & 0xf0f0f0f0u;
    auto pair = [](unsigned a, unsigned b, int i) {
        return __builtin_amdgcn_perm(__float_as_uint(float((signed char)(b >> (8 * i)))), __float_as_uint(float((signed char)(a >> (8 * i)))), 0x07060302);
    };
    const uint4 r = {pair(e, o, 0), pair(e, o, 1), pair(e, o, 2), pair(e, o, 3)};
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ bf16x8 minus24() { return __builtin_bit_cast(bf16x8, uint4{0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u}); }

// The residual stream's elements of a wave's tiles, added to its sums: all read before any is written, which the compiler cannot know to be allowed and
// would do one after the other (81 rows of 8716 outputs, 184 inputs: 15.4 us, so 8.0; 857 of 4096, 4096 inputs: 56, 46).  (m, n): of the lane's first element; past the last: the last, not stored.
template <int MB, int NC, int NT>
__device__ __forceinline__ void add_residual(const Product& p, int m, int n, f32x4 (&acc)[MB][NT]) {
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                acc[b][t][v] += ((const float*)p.out)[size_t(min(m + 16 * b + v, p.M - 1)) * p.N + min(n + 16 * t, p.N - 1)];
}

// Few rows.  A wave takes 16 NT outputs and an NW-th of the inputs in steps of 128 and asks for codes PF steps ahead (the compiler's waits, one for all ways that lead
// to a step, leave the newest load or none of them on its way, so the waves of a compute unit cover the rest); a lane's 16 bytes of a row's codes
// are 32 inputs of it.  Groups of 128: the four lanes of a row multiply their first eight, second eight .. at once.  Shorter groups: the
// lanes exchange words first, so that a product's 32 inputs lie in one group.  The activations of R rows lie in LDS, in pieces of eight in the order
// of the codes: loads come back in order, and one of a row's that waits behind the codes would take their depth away.  They are brought for
// `held` steps at a time, all of them where they fit.  Measured: one row, gate and up of 14336 outputs and 4096 inputs, 14.4 us, 4.2 TB/s of 60.6 MB
// (a plain read of as many bytes takes 10 us); 28672 outputs 13.1 us; 4096 outputs of 14336 inputs 8.6 us.  With the rows read from memory where they
// are used instead: 17.6 us.
template <typename T, bool SW, int R, int NT, int GS, int NW, int PF>
__global__ void __launch_bounds__(64 * NW, sizeof(T) == 2 ? 4 : 2)
w4_rows_kernel(Product p, int held) {
    constexpr int TERMS = Terms<T>::N, NC = SW ? NT / 2 : NT, PER = 128 / GS, MFMAS = 4 / PER;   // NC: tiles of outputs; PER: groups a step
    constexpr bool OFFSET = sizeof(T) == 2;
    static_assert(!SW || NT % 2 == 0, "gate and up side by side");
    __shared__ float part[NW][NT][4][64];
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];     // [step][term][16 pieces][R rows] of 16 bytes
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g4 = lane >> 4;
    const int n0 = blockIdx.x * (16 * NC), m0 = blockIdx.y * R;
    const int steps = (p.K + 127) / 128;
    // Rows past the last: the last, not stored; codes and scales past a row's end: its last, whose activations are zero.
    const unsigned char* const base[2] = {p.w + size_t(n0) * p.row_bytes, SW ? p.w2 + size_t(n0) * p.row_bytes : nullptr};
    const T* const sbase[2] = {(const T*)p.s + n0, SW ? (const T*)p.s2 + n0 : nullptr};
    unsigned row[NC], place[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        place[t] = min(n0 + 16 * t + n16, p.N - 1) - n0;
        row[t] = place[t] * p.row_bytes;
    }
    uint4 w[PF][NT];
    T s[PF][NT][PER];
    auto load = [&](int f, int i) {
        const unsigned at = min(i * 64 + g4 * 16, p.row_bytes - 16);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            w[f][t] = *(const uint4*)(base[t / NC] + (row[t % NC] + at));
#pragma unroll
            for (int g = 0; g < PER; ++g) s[f][t][g] = (sbase[t / NC] + size_t(min(i * PER + g, p.groups - 1)) * p.N)[place[t % NC]];
        }
    };
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](int f, int i, int first, int last) {
        bf16x8 x[TERMS][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < TERMS; ++q)
                x[q][j] = *(const bf16x8*)(lds + ((((i - first) * TERMS + q) * 16 + (GS == 128 ? 4 * g4 + j : 4 * j + g4)) * R + n16 % R) * 16);
        if constexpr (GS < 128)
#pragma unroll
            for (int t = 0; t < NT; ++t) w[f][t] = transposed(w[f][t]);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            f32x4 begin = {0.f, 0.f, 0.f, 0.f};
            if constexpr (OFFSET)
#pragma unroll
                for (int j = g * MFMAS; j < (g + 1) * MFMAS; ++j) begin = mfma16(x[0][j], minus24(), begin);
            f32x4 sum[NT];
#pragma unroll
            for (int j = g * MFMAS; j < (g + 1) * MFMAS; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const bf16x8 o = operand<T>(word(w[f][t], j));
#pragma unroll
                    for (int q = TERMS - 1; q >= 0; --q) sum[t] = mfma16(x[q][j], o, j == g * MFMAS && q == TERMS - 1 ? begin : sum[t]);
                }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float sc = float(s[f][t][g]) * (OFFSET ? 1.f : 0.0625f);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[t][v] = __builtin_fmaf(sum[t][v], sc, acc[t][v]);
            }
        }
        load(f, min(i + PF, last - 1));
    };
    for (int first = 0; first < steps; first += held) {
        const int n = min(held, steps - first), i0 = first + n * wave / NW, i1 = first + n * (wave + 1) / NW;
        if (i0 < i1)
#pragma unroll
            for (int f = 0; f < PF; ++f) load(f, min(i0 + f, i1 - 1));
        if (first) __syncthreads();
        for (int i = threadIdx.x; i < n * 16 * R; i += 64 * NW) {
            const int r = i / (n * 16), c = i % (n * 16), k = first * 128 + c * 8;          // neighbouring pieces of a row
            const T* const from = (const T*)p.a + size_t(min(m0 + r, p.M - 1)) * p.K + min(k, p.K - 8);
            unsigned char* const to = lds + ((c / 16 * TERMS * 16 + c % 16) * R + r) * 16;
            if constexpr (TERMS == 1) {
                *(bf16x8*)to = in_order(k < p.K ? *(const uint4*)from : uint4{0, 0, 0, 0});
            } else {
                const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
                bf16x8 x[TERMS];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float y = k < p.K ? (e < 4 ? lo[e] : hi[e - 4]) : 0.f;
#pragma unroll
                    for (int q = 0; q < TERMS; ++q) { x[q][e] = q + 1 < TERMS ? finite_term(y) : bf16_t(y); y -= float(x[q][e]); }
                }
#pragma unroll
                for (int q = 0; q < TERMS; ++q) *(bf16x8*)(to + q * 16 * R * 16) = x[q];
            }
        }
        __syncthreads();
        for (int i = i0; i < i1; i += PF)
#pragma unroll
            for (int f = 0; f < PF; ++f)
                if (i + f < i1) step(f, i + f, first, i1);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) part[wave][t][v][lane] = acc[t][v];
    __syncthreads();
    // the waves' parts in their order; D[4 g4 + v][n16]
    for (int i = threadIdx.x; i < NC * 16 * R; i += 64 * NW) {
        const int r = i / (NC * 16), c = i % (NC * 16), t = c / 16, l = r / 4 * 16 + c % 16, v = r % 4;
        const int m = m0 + r, n = n0 + c;
        float y = 0.f, y2 = 0.f;
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            y += part[q][t][v][l];
            if constexpr (SW) y2 += part[q][t + NC][v][l];
        }
        if (m >= p.M || n >= p.N) continue;
        const size_t at = size_t(m) * p.N + n;
        if constexpr (SW) ((T*)p.out)[at] = silu_product<T>(y, y2);
        else if (p.epi == EPI_RESIDUAL_F32) ((float*)p.out)[at] += y;
        else ((float*)p.out)[at] = y;
    }
}

// Many rows (bfloat16).  A workgroup takes 16 MB rows, 64 NC outputs and a range of the inputs; its waves take 16 NC outputs each, whose codes come
// straight into registers, a step of 128 inputs ahead and more, and are converted once for all rows.  The activations are shared: through LDS, two
// tiles, rows of 256 bytes whose 16-byte pieces lie at piece ^ row, so that 16 rows' pieces of one number lie in different banks.  Who brings a
// piece also adds up its activations, for -24 times the sum of a row's group: where a group's sum begins.
// A unit is a group of a tile of 16 outputs.  While its products run, the next unit's codes are converted and the last one's sums scaled.
// Bound by the time from a load to its use: a launch's workgroups live for a few steps, a turn's first step also waits for the codes that the step before has just
// asked for (all ways to the loop's beginning have one wait), and the ranges are joined by a second launch (3 to 4 us).
// Measured: 33 rows, 4096 outputs of 14336 inputs, groups of 64: 19.2 us, 1.6 TB/s.
template <bool SW, int MB, int NT, int GS, int WS, int XS>
__device__ __forceinline__ void w4_tile(const Product& p, unsigned char* lds, int mt, int n_begin, int split, int splits) {
    constexpr int NC = SW ? NT / 2 : NT, PER = 128 / GS, MF = 4 / PER, UNITS = PER * NT, TILE = MB * 16 * 256, SUMS = PER * MB * 16 * 4;
    constexpr int SS = WS < 2 ? 2 : WS, TURNS = WS > 2 ? WS : 2;      // sets of scales; steps until the sets come round
    static_assert(TURNS % 2 == 0 && TURNS % XS == 0, "a step's sets are known when it is compiled");
    static_assert(!SW || NT % 2 == 0, "gate and up side by side");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g4 = lane >> 4;
    const int m0 = mt * (16 * MB), n0 = n_begin + wave * (16 * NC);
    const int steps = (p.K + 127) / 128, i0 = int(int64_t(steps) * split / splits), i1 = int(int64_t(steps) * (split + 1) / splits);
    // codes and scales from the wave's first row on: offsets of 32 bits
    const int n_first = min(n0, p.N - 1);
    const unsigned char* const base[2] = {p.w + size_t(n_first) * p.row_bytes, SW ? p.w2 + size_t(n_first) * p.row_bytes : nullptr};
    const bf16_t* const sbase[2] = {(const bf16_t*)p.s + n_first, SW ? (const bf16_t*)p.s2 + n_first : nullptr};
    unsigned row[NC], place[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        place[t] = min(n0 + 16 * t + n16, p.N - 1) - n_first;
        row[t] = place[t] * p.row_bytes;
    }
    uint4 w[WS][NT];
    bf16_t s[SS][NT][PER];
    auto load_codes = [&](int f, int i, int t) { w[f][t] = *(const uint4*)(base[t / NC] + (row[t % NC] + unsigned(min(i * 64 + g4 * 16, p.row_bytes - 16)))); };
    auto load_scales = [&](int f, int i) {
#pragma unroll
        for (int g = 0; g < PER; ++g)
#pragma unroll
            for (int t = 0; t < NT; ++t) s[f][t][g] = (sbase[t / NC] + size_t(min(i * PER + g, p.groups - 1)) * p.N)[place[t % NC]];
    };
    // this thread's piece of 16 rows: from memory through registers into LDS
    const int piece = tid & 15, r0 = tid >> 4;
    const bf16_t* const abase = (const bf16_t*)p.a + size_t(m0) * p.K;
    unsigned arow[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) arow[b] = min(16 * b + r0, p.M - 1 - m0) * p.K;
    uint4 raw[XS][MB];
    auto load_rows = [&](int q, int i) {
        const int k = i * 128 + piece * 8;
#pragma unroll
        for (int b = 0; b < MB; ++b) raw[q][b] = *(const uint4*)(abase + (arow[b] + min(k, p.K - 8)));
    };
    const int put = r0 * 256 + ((piece ^ r0) << 4);
    auto stage = [&](int q, int i, int buf) {
        const unsigned keep = i * 128 + piece * 8 < p.K ? ~0u : 0u;        // inputs past the last: zeros
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            raw[q][b].x &= keep; raw[q][b].y &= keep; raw[q][b].z &= keep; raw[q][b].w &= keep;
            *(bf16x8*)(lds + buf * TILE + b * 4096 + put) = in_order(raw[q][b]);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, word(raw[q][b], e)), __builtin_bit_cast(bf16x2, 0xc1c0c1c0u), sum, false);
            sum = add_group<GS / 8>(sum);
            *(float*)(lds + 2 * TILE + buf * SUMS + ((piece / (GS / 8)) * (MB * 16) + b * 16 + r0) * 4) = sum;
        }
    };
    const int get = n16 * 256;
    auto fragment = [&](int buf, int b, int j) {
        const int c = GS == 128 ? 4 * g4 + j : 4 * j + g4;
        return *(const bf16x8*)(lds + buf * TILE + b * 4096 + get + ((c ^ n16) << 4));
    };
    f32x4 acc[MB][NT];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 o[MF];                          // the unit's codes; behind their product, the next unit's
    f32x4 sum[2][MB];
    auto convert = [&](int f, int u, int j) { o[j] = codes8(word(w[f][u % NT], u / NT * MF + j)); };
    auto begin = [&](int f, int u) {
#pragma unroll
        for (int b = 0; b < MB; ++b) sum[u & 1][b] = *(const f32x4*)(lds + 2 * TILE + f * SUMS + (u / NT * (MB * 16) + b * 16 + 4 * g4) * 4);
    };
    auto scaled = [&](int f, int u) {
        const float sc = float(s[f][u % NT][u / NT]);
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[b][u % NT][v] = __builtin_fmaf(sum[u & 1][b][v], sc, acc[b][u % NT][v]);
    };
    auto step = [&](auto odd, int i) {
        constexpr int turn = decltype(odd)::value, f = turn % 2, fw = turn % WS, fs = turn % SS, q = (turn + 1) % XS;   // turn: (i - i0) % TURNS
        // no branches: what a step past the last would need is loaded from the last, and not used
        stage(q, i + 1, f ^ 1);
        load_rows(q, min(i + 1 + XS, i1 - 1));
        if constexpr (GS < 128)
#pragma unroll
            for (int t = 0; t < NT; ++t) w[fw][t] = transposed(w[fw][t]);
        bf16x8 x[MB][MF];
        begin(f, 0);
#pragma unroll
        for (int j = 0; j < MF; ++j) convert(fw, 0, j);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int g = u / NT, t = u % NT;
            if (t == 0)
#pragma unroll
                for (int j = 0; j < MF; ++j)
#pragma unroll
                    for (int b = 0; b < MB; ++b) x[b][j] = fragment(f, b, g * MF + j);
            __builtin_amdgcn_sched_barrier(0);
            if (u > 0) scaled(fs, u - 1);
#pragma unroll
            for (int j = 0; j < MF; ++j) {
#pragma unroll
                for (int b = 0; b < MB; ++b) sum[u & 1][b] = mfma16(x[b][j], o[j], sum[u & 1][b]);
                if (u + 1 < UNITS) convert(fw, u + 1, j);
            }
            if (u + 1 < UNITS) begin(f, u + 1);
            if (g == PER - 1) load_codes(fw, min(i + WS, i1 - 1), t);
            __builtin_amdgcn_sched_barrier(0);
        }
        scaled(fs, UNITS - 1);
        load_scales(fs, min(i + SS, i1 - 1));
        __syncthreads();
    };
    if (i0 < i1) {
#pragma unroll
        for (int q = 0; q < (SS > XS + 1 ? SS : XS + 1); ++q) {
            const int i = min(i0 + q, i1 - 1);
            if (q < WS)
#pragma unroll
                for (int t = 0; t < NT; ++t) load_codes(q, i, t);
            if (q < SS) load_scales(q, i);
            if (q <= XS) load_rows(q % XS, i);
            if (q == 0) stage(0, i0, 0);
        }
    }
    __syncthreads();
    for (int i = i0; i < i1; i += TURNS) {
        step(std::integral_constant<int, 0>{}, i);
        if (i + 1 < i1) step(std::integral_constant<int, 1>{}, i + 1);
        if constexpr (TURNS == 4) {
            if (i + 2 < i1) step(std::integral_constant<int, 2>{}, i + 2);
            if (i + 3 < i1) step(std::integral_constant<int, 3>{}, i + 3);
        }
    }
    if (!SW && splits == 1 && p.epi == EPI_RESIDUAL_F32) add_residual<MB, NC>(p, m0 + 4 * g4, n0 + n16, acc);
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int m = m0 + 16 * b + 4 * g4 + v, n = n0 + 16 * t + n16;
                if (m >= p.M || n >= p.N) continue;
                const size_t at = size_t(m) * p.N + n;
                if (splits > 1) {
                    float* d = p.parts + size_t(split) * (SW ? 2 : 1) * p.M * p.N + at;
                    *d = acc[b][t][v];
                    if constexpr (SW) d[size_t(p.M) * p.N] = acc[b][t + NC][v];
                } else if constexpr (SW) ((bf16_t*)p.out)[at] = silu_product<bf16_t>(acc[b][t][v], acc[b][t + NC][v]);
                else ((float*)p.out)[at] = acc[b][t][v];
            }
}

// Many rows of float32 models.  As above, with three terms of each activation in LDS and two tiles of 16 rows; a code's conversion (twice a
// bfloat16 one's instructions) serves 32 rows, a fragment of activations two tiles of outputs.  Bound by those conversions and by the time of a
// step, some 1.2 us, while a launch has few workgroups (the inputs are not divided).  Measured: 732 rows, 3553 outputs, 1320 inputs: 36 us (groups of 32; of 128: 34), four
// rows at a time 206.
template <bool SW, int GS>
__global__ void __launch_bounds__(256, 2)
w4_f32_kernel(Product p) {
    constexpr int MB = 2, NT = 2, NC = SW ? 1 : 2, PER = 128 / GS, MF = 4 / PER, TERMS = Terms<float>::N;
    __shared__ __attribute__((aligned(16))) unsigned char lds[2][TERMS][MB * 16 * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g4 = lane >> 4;
    const int m0 = blockIdx.y * (16 * MB), n0 = blockIdx.x * (64 * NC) + wave * (16 * NC), steps = (p.K + 127) / 128;
    const int n_first = min(n0, p.N - 1);
    const unsigned char* const base[2] = {p.w + size_t(n_first) * p.row_bytes, SW ? p.w2 + size_t(n_first) * p.row_bytes : nullptr};
    const float* const sbase[2] = {(const float*)p.s + n_first, SW ? (const float*)p.s2 + n_first : nullptr};
    unsigned row[NC], place[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        place[t] = min(n0 + 16 * t + n16, p.N - 1) - n_first;
        row[t] = place[t] * p.row_bytes;
    }
    uint4 w[2][NT];
    float s[2][NT][PER];
    auto load = [&](int f, int i) {
        const unsigned at = min(i * 64 + g4 * 16, p.row_bytes - 16);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            w[f][t] = *(const uint4*)(base[t / NC] + (row[t % NC] + at));
#pragma unroll
            for (int g = 0; g < PER; ++g) s[f][t][g] = (sbase[t / NC] + size_t(min(i * PER + g, p.groups - 1)) * p.N)[place[t % NC]];
        }
    };
    const int piece = tid & 15, r0 = tid >> 4, put = r0 * 256 + ((piece ^ r0) << 4);
    const float* from[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) from[b] = (const float*)p.a + size_t(min(m0 + 16 * b + r0, p.M - 1)) * p.K;
    f32x4 raw[MB][2];
    auto load_rows = [&](int i) {
        const int k = i * 128 + piece * 8, at = min(k, p.K - 8);
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) raw[b][h] = *(const f32x4*)(from[b] + at + 4 * h);
    };
    auto stage = [&](int i, int buf) {
        const bool keep = i * 128 + piece * 8 < p.K;            // inputs past the last: zeros
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = keep ? raw[b][e / 4][e % 4] : 0.f;
#pragma unroll
            for (int q = 0; q < TERMS; ++q) {
                bf16x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) { x[e] = q + 1 < TERMS ? finite_term(y[e]) : bf16_t(y[e]); y[e] -= float(x[e]); }
                *(bf16x8*)(lds[buf][q] + b * 4096 + put) = x;
            }
        }
    };
    f32x4 acc[MB][NT];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](auto f_, int i) {
        constexpr int f = decltype(f_)::value;
        stage(i + 1, f ^ 1);
        load_rows(min(i + 2, steps - 1));
        load(f ^ 1, min(i + 1, steps - 1));
        if constexpr (GS < 128)
#pragma unroll
            for (int t = 0; t < NT; ++t) w[f][t] = transposed(w[f][t]);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            f32x4 sum[MB][NT];
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = g * MF; j < (g + 1) * MF; ++j) {
                const int c = GS == 128 ? 4 * g4 + j : 4 * j + g4;
                bf16x8 o[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) o[t] = operand<float>(word(w[f][t], j));
#pragma unroll
                for (int q = TERMS - 1; q >= 0; --q)
#pragma unroll
                    for (int b = 0; b < MB; ++b) {
                        const bf16x8 x = *(const bf16x8*)(lds[f][q] + b * 4096 + n16 * 256 + ((c ^ n16) << 4));
#pragma unroll
                        for (int t = 0; t < NT; ++t) sum[b][t] = mfma16(x, o[t], sum[b][t]);
                    }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float sc = s[f][t][g] * 0.0625f;
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[b][t][v] = __builtin_fmaf(sum[b][t][v], sc, acc[b][t][v]);
            }
        }
        __syncthreads();
    };
    load(0, 0);
    load_rows(0);
    stage(0, 0);
    load_rows(min(1, steps - 1));
    __syncthreads();
    for (int i = 0; i < steps; i += 2) {
        step(std::integral_constant<int, 0>{}, i);
        if (i + 1 < steps) step(std::integral_constant<int, 1>{}, i + 1);
    }
    if (!SW && p.epi == EPI_RESIDUAL_F32) add_residual<MB, NC>(p, m0 + 4 * g4, n0 + n16, acc);
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int m = m0 + 16 * b + 4 * g4 + v, n = n0 + 16 * t + n16;
                if (m >= p.M || n >= p.N) continue;
                float* const d = (float*)p.out + size_t(m) * p.N + n;
                if constexpr (SW) *d = silu_product<float>(acc[b][t][v], acc[b][t + NC][v]);
                else *d = acc[b][t][v];
            }
}

// Workgroups are dealt out to the eight XCDs in turn.  A column (the row tiles of the same outputs and inputs) stays on one, so that they share its
// L2; neighbouring columns go to different ones.
struct Place { int column, mt; };
__device__ __forceinline__ Place place_of(int b, int m_tiles) {
    const int slot = b / 8;
    return {slot / m_tiles * 8 + b % 8, slot % m_tiles};
}
inline int blocks_of(int columns, int m_tiles) { return (columns + 7) / 8 * 8 * m_tiles; }

template <bool SW, int MB, int NT, int GS, int WS, int XS>
__global__ void __launch_bounds__(256, 2)
w4_tile_kernel(Product p, int m_tiles, int n_tiles, int splits) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const Place at = place_of(blockIdx.x, m_tiles);
    if (at.column < n_tiles * splits) w4_tile<SW, MB, NT, GS, WS, XS>(p, lds, at.mt, at.column % n_tiles * (64 * (SW ? NT / 2 : NT)), at.column / n_tiles, splits);
}

// ---- many rows
// The weights enter as code times scale in half precision: eleven bits, exact.  For that an output's scales are taken in units of 2^E, the
// largest of them in [2^10, 2^11), and a row's activations in units that put the largest in [2^14, 2^15); both are exact down to 2^-24 of a
// unit, 2^-35 of the largest scale, 2^-39 of the largest activation.  A pass before the product finds the units, and lays the activations
// out as the product brings them into LDS: [64 inputs][row][eight pieces of eight], the pieces in the order in which a product's lanes take them, swizzled.
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
__device__ __forceinline__ f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

struct Wide {
    Product p;
    _Float16* x;            // [2 steps][m_pad][64]
    int* row_unit;          // [m_pad]: exponents of the units
    int* out_unit;          // [2][N]
    int m_pad, shift;       // 2^shift inputs share a scale
};
__device__ __forceinline__ float power(int biased) { return __uint_as_float(unsigned(biased) << 23); }

// Workgroups for 64 outputs each, then for a row each, which is kept in registers between its largest magnitude and its place (up to 16384 inputs).
__global__ void __launch_bounds__(256)
w4_prepare_kernel(Wide q) {
    constexpr int HELD = 8;
    __shared__ unsigned top[256];
    const Product& p = q.p;
    const int tid = threadIdx.x, per = (p.N + 63) / 64, of_outputs = (p.s2 ? 2 : 1) * per;
    unsigned most = 0;                                          // as bits: magnitudes order like the numbers; infinities and NaN do not count
    if (int(blockIdx.x) < of_outputs) {
        const int which = blockIdx.x / per, n = int(blockIdx.x) % per * 64 + (tid & 63);
        const unsigned short* const s = (const unsigned short*)(which ? p.s2 : p.s) + min(n, p.N - 1);
#pragma unroll 16
        for (int g = tid >> 6; g < p.groups; g += 4) {
            const unsigned v = s[size_t(g) * p.N] & 0x7fffu;
            most = max(most, v < 0x7f80u ? v : 0u);
        }
        top[tid] = most;
        __syncthreads();
        if (tid < 64 && n < p.N) q.out_unit[which * p.N + n] = max(int(max(max(most, top[tid + 64]), max(top[tid + 128], top[tid + 192])) >> 7), 11) - 137;
        return;
    }
    const int m = int(blockIdx.x) - of_outputs, chunks = (p.K + 127) / 128 * 16;
    const bf16_t* const row = (const bf16_t*)p.a + size_t(min(m, p.M - 1)) * p.K;
    auto read = [&](int c) { return 8 * c < p.K && m < p.M ? *(const uint4*)(row + 8 * c) : uint4{0, 0, 0, 0}; };
    auto largest = [&](uint4 v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned lo = word(v, e) & 0x7fffu, hi = word(v, e) >> 16 & 0x7fffu;
            most = max(most, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
        }
    };
    uint4 held[HELD];
#pragma unroll
    for (int r = 0; r < HELD; ++r) held[r] = read(tid + 256 * r);
#pragma unroll
    for (int r = 0; r < HELD; ++r) largest(held[r]);
    for (int c = tid + 256 * HELD; c < chunks; c += 256) largest(read(c));
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, unsigned(__shfl_xor(int(most), d)));
    if ((tid & 63) == 0) top[tid >> 6] = most;
    __syncthreads();
    const int e = max(int(max(max(top[0], top[1]), max(top[2], top[3])) >> 7), 15);
    const float f = power(268 - e);                             // 2^(14 - (e - 127))
    if (tid == 0) q.row_unit[m] = e - 141;
    auto put = [&](int c, uint4 v) {
        const int k = 8 * c, r = k & 127, slot = ((r >> 3 & 1) * 4 + (r >> 5)) ^ (m >> 1 & 7);
        f16x8 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                           // elements i and i + 4
            const unsigned a = word(v, i >> 1), b = word(v, 2 + (i >> 1));
            h[2 * i] = _Float16(__uint_as_float(i & 1 ? a & 0xffff0000u : a << 16) * f);
            h[2 * i + 1] = _Float16(__uint_as_float(i & 1 ? b & 0xffff0000u : b << 16) * f);
        }
        *(f16x8*)(q.x + (size_t((k >> 7) * 2 + (r >> 4 & 1)) * q.m_pad + m) * 64 + slot * 8) = h;
    };
#pragma unroll
    for (int r = 0; r < HELD; ++r)
        if (tid + 256 * r < chunks) put(tid + 256 * r, held[r]);
    for (int c = tid + 256 * HELD; c < chunks; c += 256) put(c, read(c));
}

// Eight codes of a word times a scale: 16 + the code's four bits (the upper one turned) is 24 + c, and one multiply-add makes (24 + c) s - 24 s of it, exact.
// s: the scale and -24 times it.
__device__ __forceinline__ f16x8 weights8(unsigned w, f16x2 s) {
    constexpr unsigned M = 0x03c003c0u, B = 0x4e004e00u;
    auto pair = [&](unsigned y) { return __builtin_bit_cast(unsigned, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (y & M) ^ B), f16x2{s[0], s[0]}, f16x2{s[1], s[1]})); };
    const uint4 r = {pair(w << 6), pair(w << 2), pair(w >> 2), pair(w >> 6)};
    return __builtin_bit_cast(f16x8, r);
}

// A workgroup takes 16 MB rows and 64 NC outputs (SwiGLU: of each matrix), a wave all of the rows and 16 NC outputs.  Activations come into LDS in
// halves of a step, a ring of RING, by loads that pass no register; codes into registers, steps ahead.  Half-way through a half step all its
// operands are read: there the waves meet, the next half must have come, and the last of the ring is asked for, into the place of the half before.
// Loads come back in order, so the ring has to reach as far ahead as the codes; a turn of the loop begins with a wait for its first codes, which takes in loads of the
// half step before.  Measured: 1024 rows, 10240 outputs of 8192 inputs: 147 us, 1.17 PFLOP/s, of the 1.20 that a library's large bfloat16 product reaches
// here; 10 us more for the pass before (157 for both under the profiler, the call without it 154).
#define CAKE_LDS_AS __attribute__((address_space(3)))
template <bool SW, int MB, int NT>
__device__ __forceinline__ void w4_wide_tile(const Wide& q, unsigned char* lds, int mt, int n_begin, int split, int splits) {
    constexpr int NC = SW ? NT / 2 : NT, STAGE = MB * 2048, DMA = MB / 2, WS = MB < 8 ? 4 : 2, RING = 4;   // WS: steps of codes on their way
    static_assert(!SW || NT % 2 == 0, "gate and up side by side");
    static_assert(MB % 2 == 0, "a stage in whole loads of each wave");
    const Product& p = q.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g4 = lane >> 4;
    const int m0 = mt * (16 * MB), n0 = n_begin + wave * (16 * NC), n_first = min(n0, p.N - 1);
    const int steps = (p.K + 127) / 128, i0 = int(int64_t(steps) * split / splits), i1 = int(int64_t(steps) * (split + 1) / splits), h1 = 2 * i1;
    const unsigned char* const base[2] = {p.w + size_t(n_first) * p.row_bytes, SW ? p.w2 + size_t(n_first) * p.row_bytes : nullptr};
    const __amdgpu_buffer_rsrc_t sbase[2] = {__builtin_amdgcn_make_buffer_rsrc((void*)p.s, 0, p.groups * p.N * 2, 0x00020000),
                                             __builtin_amdgcn_make_buffer_rsrc((void*)(SW ? p.s2 : p.s), 0, p.groups * p.N * 2, 0x00020000)};
    unsigned row[NC], place[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        place[t] = min(n0 + 16 * t + n16, p.N - 1) - n_first;
        row[t] = place[t] * p.row_bytes;
    }
    auto unit_of = [&](int t) { return q.out_unit[(t / NC) * p.N + n_first + place[t % NC]]; };
    float per_unit[NT];                                         // what a scale is multiplied by
#pragma unroll
    for (int t = 0; t < NT; ++t) per_unit[t] = power(127 - unit_of(t));
    uint4 w[WS][NT];
    unsigned short s[WS][NT];
    auto load = [&](int f, int i) {
        const unsigned at = min(i * 64 + g4 * 16, p.row_bytes - 16);
        const int g = min((i * 128 + g4 * 32) >> q.shift, p.groups - 1) * p.N + n_first;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            w[f][t] = *(const uint4*)(base[t / NC] + (row[t % NC] + at));
            s[f][t] = __builtin_amdgcn_raw_buffer_load_b16(sbase[t / NC], (g + place[t % NC]) * 2, 0, 0);
        }
    };
    // buffer loads: the compiler counts them as what they are, where it waits for loads into registers
    const __amdgpu_buffer_rsrc_t xs = __builtin_amdgcn_make_buffer_rsrc(q.x, 0, steps * 256 * q.m_pad, 0x00020000);
    const int x_from = wave * (DMA * 1024) + lane * 16;
    auto bring = [&](int h) {                                   // half step h into its place in the ring
        const int from = (min(h, h1 - 1) * q.m_pad + m0) * 128;
        CAKE_LDS_AS void* const to = (CAKE_LDS_AS void*)(lds + h % RING * STAGE + wave * (DMA * 1024));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, to, 16, x_from, from, 0, 0);
        if constexpr (DMA > 1) __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, to, 16, x_from, from, 1024, 0);
        if constexpr (DMA > 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, to, 16, x_from, from, 2 * 1024, 0);
        if constexpr (DMA > 3) __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, to, 16, x_from, from, 3 * 1024, 0);
    };
    const int get[2] = {n16 * 128 + ((g4 ^ (n16 >> 1 & 7)) << 4), n16 * 128 + (((4 + g4) ^ (n16 >> 1 & 7)) << 4)};
    f32x4 acc[MB][NT];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    f16x8 x[MB];
    f16x2 sc[NT];
    auto scales = [&](int f) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const _Float16 y = _Float16(__uint_as_float(unsigned(s[f][t]) << 16) * per_unit[t]);
            sc[t] = f16x2{y, y * _Float16(-24.f)};
        }
    };
    // The products of eight inputs a lane, word j of the codes; behind the last tile's, the operands of what follows.
    auto products = [&](int f, int j, int stage, int half) {
        f16x8 o = weights8(word(w[f][0], j), sc[0]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f16x8 next;
            if (t + 1 < NT) next = weights8(word(w[f][t + 1 < NT ? t + 1 : t], j), sc[t + 1 < NT ? t + 1 : t]);
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                acc[b][t] = mfma16h(x[b], o, acc[b][t]);
                if (t == NT - 1) x[b] = *(const f16x8*)(lds + stage * STAGE + b * 2048 + get[half]);
            }
            o = next;
        }
    };
    // The waits for the ring count what has been asked for since: the order of the loads is held, and check_lds_loads.py follows the listing's paths.
    if (i0 < i1) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < RING - 1; ++h) bring(2 * i0 + h);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < WS; ++f) load(f, min(i0 + f, i1 - 1));
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NT * WS + (RING - 2) * DMA) : "memory");
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int b = 0; b < MB; ++b) x[b] = *(const f16x8*)(lds + 2 * i0 % RING * STAGE + b * 2048 + get[0]);
        // Behind the half step that must have come the next one was asked for and, while steps go on, a step's codes and scales (2 NT).  Of the last
        // steps (more_ false) those are used by nobody, and the compiler drops them: there the next half step alone may be outstanding.
        auto step = [&](auto f_, auto more_, int i) {
            constexpr int f = decltype(f_)::value, CODES = decltype(more_)::value ? 2 * NT : 0;
            scales(f);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int h = 2 * i + half;
                products(f, 2 * half, h % RING, 1);
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 3) * DMA + CODES) : "memory");
                __builtin_amdgcn_s_barrier();
                bring(h + RING - 1);
                __builtin_amdgcn_sched_barrier(0);
                products(f, 2 * half + 1, (h + 1) % RING, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (CODES > 0) load(f, min(i + WS, i1 - 1));
            __builtin_amdgcn_sched_barrier(0);
        };
        const std::true_type more{};
        const std::false_type last{};
        int i = i0;
        for (; i + WS <= i1; i += WS) {
            step(std::integral_constant<int, 0>{}, more, i);
            step(std::integral_constant<int, 1>{}, more, i + 1);
            if constexpr (WS == 4) {
                step(std::integral_constant<int, 2>{}, more, i + 2);
                step(std::integral_constant<int, 3>{}, more, i + 3);
            }
        }
        if (i < i1) step(std::integral_constant<int, 0>{}, last, i);
        if constexpr (WS == 4) {
            if (i + 1 < i1) step(std::integral_constant<int, 1>{}, last, i + 1);
            if (i + 2 < i1) step(std::integral_constant<int, 2>{}, last, i + 2);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // what was asked for past the end
    }
    int unit[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) unit[t] = unit_of(t);
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int4 ru = *(const int4*)(q.row_unit + m0 + 16 * b + 4 * g4);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[b][t][v] = ldexpf(acc[b][t][v], (v == 0 ? ru.x : v == 1 ? ru.y : v == 2 ? ru.z : ru.w) + unit[t]);
    }
    if (!SW && splits == 1 && p.epi == EPI_RESIDUAL_F32) add_residual<MB, NC>(p, m0 + 4 * g4, n0 + n16, acc);
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NC; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int m = m0 + 16 * b + 4 * g4 + v, n = n0 + 16 * t + n16;
                if (m >= p.M || n >= p.N) continue;
                const size_t at = size_t(m) * p.N + n;
                if (splits > 1) {
                    float* d = p.parts + size_t(split) * (SW ? 2 : 1) * p.M * p.N + at;
                    *d = acc[b][t][v];
                    if constexpr (SW) d[size_t(p.M) * p.N] = acc[b][t + NC][v];
                } else if constexpr (SW) ((bf16_t*)p.out)[at] = silu_product<bf16_t>(acc[b][t][v], acc[b][t + NC][v]);
                else ((float*)p.out)[at] = acc[b][t][v];
            }
}

// Workgroups of two widths, so that a launch fills the compute units evenly: the first `more` of a row tile's `tiles` take 64 outputs more than the others.
template <bool SW, int MB, int NT>
__global__ void __launch_bounds__(256, 2)
w4_wide_kernel(Wide q, int m_tiles, int tiles, int more, int splits) {
    constexpr int U = SW ? 2 : 1, W = 64 * NT / U;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const Place at = place_of(blockIdx.x, m_tiles);
    if (at.column >= tiles * splits) return;
    const int tile = at.column % tiles, split = at.column / tiles;
    if constexpr (NT < 4)
        if (tile < more) {
            w4_wide_tile<SW, MB, NT + U>(q, lds, at.mt, tile * (W + 64), split, splits);
            return;
        }
    w4_wide_tile<SW, MB, NT>(q, lds, at.mt, tile * W + more * 64, split, splits);
}

// The ranges' parts in their order.
template <bool SW>
__global__ void __launch_bounds__(256)
w4_parts_kernel(Product p, int splits) {
    const size_t size = size_t(p.M) * p.N, stride = SW ? 2 * size : size;
    for (size_t i = size_t(blockIdx.x) * 256 + threadIdx.x; i < size; i += size_t(gridDim.x) * 256) {
        float y = 0.f, y2 = 0.f;
#pragma unroll 8
        for (int q = 0; q < splits; ++q) {
            y += p.parts[q * stride + i];
            if constexpr (SW) y2 += p.parts[q * stride + size + i];
        }
        if constexpr (SW) ((bf16_t*)p.out)[i] = silu_product<bf16_t>(y, y2);
        else if (p.epi == EPI_RESIDUAL_F32) ((float*)p.out)[i] += y;
        else ((float*)p.out)[i] = y;
    }
}

// A lane takes eight weights of a row, the lanes of a group find its largest magnitude; a workgroup takes the same group of neighbouring rows,
// whose scales lie side by side.  Bound by the bytes.
template <typename T, int GS>
__global__ void __launch_bounds__(256)
pack_w4_kernel(const T* __restrict__ w, unsigned char* __restrict__ codes, T* __restrict__ scales, T* __restrict__ values, int N, int K, int row_bytes, int groups) {
    constexpr int LANES = GS / 8, ROWS = 256 / LANES;
    const int64_t blocks = int64_t((N + ROWS - 1) / ROWS) * groups;
    for (int64_t i = blockIdx.x; i < blocks; i += gridDim.x) {
        const int group = int(i % groups), n = int(i / groups) * ROWS + threadIdx.x / LANES, piece = group * LANES + threadIdx.x % LANES, k = piece * 8;
        if (n >= N) continue;                             // whole groups of lanes
        float x[8] = {};
        if (k < K) {
            const T* from = w + size_t(n) * K + k;
            if constexpr (sizeof(T) == 2) {
                const bf16x8 v = *(const bf16x8*)from;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = float(v[e]);
            } else {
                const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[e] = lo[e]; x[e + 4] = hi[e]; }
            }
        }
        unsigned m = 0;      // magnitudes as bits: they order like the numbers, infinities and NaN on top
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) m = max(m, unsigned(__shfl_xor(int(m), d)));
        const T s = T(m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(m) / 7.f);
        const float scale = float(s);
        if (piece % LANES == 0) scales[size_t(group) * N + n] = s;
        if (piece * 4 >= row_bytes) continue;
        unsigned packed = 0;
        float c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            c[e] = scale > 0.f ? fminf(fmaxf(rintf(x[e] / scale), -7.f), 7.f) : 0.f;
            packed |= (unsigned(int(c[e])) & 15u) << (4 * e);
            c[e] *= scale;
        }
        *(unsigned*)(codes + size_t(n) * row_bytes + piece * 4) = packed;
        if (values && k < K) {
            T* d = values + size_t(n) * K + k;
            if constexpr (sizeof(T) == 2) {
                bf16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = bf16_t(c[e]);
                *(bf16x8*)d = v;
            } else {
                *(f32x4*)d = f32x4{c[0], c[1], c[2], c[3]};
                *(f32x4*)(d + 4) = f32x4{c[4], c[5], c[6], c[7]};
            }
        }
    }
}

// Waves that share a workgroup's inputs.  Bytes on their way are waves times the codes each has asked for: where a launch has workgroups
// enough, fewer waves with longer ways waste less on beginning and joining; where it has few and the inputs are long, more waves.  One row, 4 / 8 / 16
// waves, us: 28672 outputs of 4096 inputs 13.1 / 15.1 / -, 8192 of 4096 7.0 / 6.3 / 6.5, 4096 of 14336 17.2 / 11.3 / 9.6.
template <typename T, bool SW, int GS>
hipError_t rows(const Product& p, hipStream_t st) {
    constexpr int NT = SW ? 2 : 1;
    auto go = [&](auto r, auto nw) {
        constexpr int R = decltype(r)::value, PF = sizeof(T) == 2 ? 2 : 1, NW = decltype(nw)::value, STEP = Terms<T>::N * 256 * R;
        const int held = std::min((p.K + 127) / 128, (sizeof(T) == 2 ? 32 << 10 : 24 << 10) / STEP);
        // a grid's second size, at most 65535: `choose` sends fewer than 2^16 fours of rows here, whatever their outputs and inputs
        hipLaunchKernelGGL((w4_rows_kernel<T, SW, R, NT, GS, NW, PF>), dim3(unsigned((p.N + 15) / 16), unsigned((p.M + R - 1) / R)), dim3(64 * NW), held * STEP, st, p, held);
        return hipGetLastError();
    };
    auto by_waves = [&](auto r) {
        const std::integral_constant<int, 8> eight{};
        if constexpr (sizeof(T) == 4) return go(r, eight);
        else {
            const int n = (p.N + 15) / 16 * NT;
            return n > 1024 ? go(r, std::integral_constant<int, 4>{}) : n > 256 || p.K < 8192 ? go(r, eight) : go(r, std::integral_constant<int, 16>{});
        }
    };
    return p.M == 1 ? by_waves(std::integral_constant<int, 1>{}) : by_waves(std::integral_constant<int, 4>{});
}

template <bool SW>
hipError_t add_parts(const Product& p, int splits, hipStream_t st) {
    hipLaunchKernelGGL(w4_parts_kernel<SW>, dim3(unsigned(std::min<int64_t>((int64_t(p.M) * p.N + 255) / 256, 1 << 16))), dim3(256), 0, st, p, splits);
    return hipGetLastError();
}
// How many parts of the result the workspace holds.
inline int64_t parts_in(size_t bytes, const Product& p) { return int64_t(bytes / (size_t(p.M) * p.N * (p.epi == EPI_SWIGLU ? 8 : 4))); }

template <bool SW, int GS>
hipError_t tiles(Product p, float* ws, size_t ws_bytes, hipStream_t st) {
    auto go = [&](auto mb, auto ahead) {
        constexpr int MB = decltype(mb)::value, NT = 2, LDS = 2 * MB * 16 * (256 + 128 / GS * 4);
        const int m_tiles = (p.M + 16 * MB - 1) / (16 * MB), n_tiles = (p.N + 64 * (SW ? 1 : 2) - 1) / (64 * (SW ? 1 : 2)), steps = (p.K + 127) / 128;
        int64_t splits = std::min<int64_t>(steps / 4, 512 / (int64_t(m_tiles) * n_tiles));
        splits = std::max<int64_t>(1, std::min(splits, parts_in(ws_bytes, p)));
        p.parts = ws;
        hipLaunchKernelGGL((w4_tile_kernel<SW, MB, NT, GS, decltype(ahead)::value, 2>), dim3(unsigned(blocks_of(int(n_tiles * splits), m_tiles))), dim3(256), LDS, st, p, m_tiles, n_tiles,
                           int(splits));
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || splits == 1 ? e : add_parts<SW>(p, int(splits), st);
    };
    const std::integral_constant<int, 1> one{};
    const std::integral_constant<int, 2> two{};
    const std::integral_constant<int, 3> three{};
    const std::integral_constant<int, 4> four{};
    return p.M <= 16 ? go(one, four) : p.M <= 32 ? go(two, four) : p.M <= 48 ? go(three, two) : go(four, two);
}

template <bool SW>
hipError_t wide(Product p, int group, float* ws, size_t ws_bytes, hipStream_t st) {
    auto go = [&](auto mb, auto nt, int tiles, int more) {
        constexpr int MB = decltype(mb)::value, NT = decltype(nt)::value, LDS = 4 * MB * 2048;
        const int m_tiles = (p.M + 16 * MB - 1) / (16 * MB), steps = (p.K + 127) / 128;
        Wide q;
        q.m_pad = m_tiles * 16 * MB;
        q.shift = group == 128 ? 7 : group == 64 ? 6 : 5;
        unsigned char* at = (unsigned char*)ws;
        q.x = (_Float16*)at; at += size_t(steps) * 2 * q.m_pad * 128;
        q.row_unit = (int*)at; at += size_t(q.m_pad) * 4;
        q.out_unit = (int*)at; at += (size_t(p.N) * (SW ? 2 : 1) * 4 + 15) / 16 * 16;
        p.parts = (float*)at;
        int64_t splits = std::min<int64_t>(steps / 24, 512 / (int64_t(m_tiles) * tiles));
        splits = std::max<int64_t>(1, std::min(splits, parts_in(ws_bytes - (at - (unsigned char*)ws), p)));
        q.p = p;
        hipLaunchKernelGGL(w4_prepare_kernel, dim3(unsigned(q.m_pad + (p.N + 63) / 64 * (SW ? 2 : 1))), dim3(256), 0, st, q);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((w4_wide_kernel<SW, MB, NT>), dim3(unsigned(blocks_of(int(tiles * splits), m_tiles))), dim3(256), LDS, st, q, m_tiles, tiles, more, int(splits));
        e = hipGetLastError();
        return e != hipSuccess || splits == 1 ? e : add_parts<SW>(p, int(splits), st);
    };
    const std::integral_constant<int, 4> four{};
    const std::integral_constant<int, 8> eight{};
    const int units = (p.N + 63) / 64, m_tiles = (p.M + 127) / 128;      // 64 outputs
    // 128 rows or 64: a workgroup's codes are converted once for its rows, but 64 make twice the workgroups, and up to 512 rows less padding.
    // 128 against 64 rows, us: 1024 rows, 10240 outputs of 8192 inputs 156 / 237; 857, 4096 of 11008 106 / 137; 640, 5120 of 5120 53.8 / 62.6; 768,
    // 4096 of 4096 45.6 / 44.6; 512, 4096 of 14336 86.8 / 89.9; 320, 14336 of 4096 71.6 / 63.6; 128, 28672 of 4096 45.3 / 50.6.
    if (int64_t(m_tiles) * units < 400 || (p.M < 512 && m_tiles * 2 != (p.M + 63) / 64)) return go(four, std::integral_constant<int, SW ? 2 : 1>{}, units, 0);
    // two workgroups a compute unit, in as few rounds as their widths allow
    const int slots = std::max(1, 512 / m_tiles), most = SW ? 2 : 4, rounds = (units + slots * most - 1) / (slots * most);
    const int tiles = std::min(units, rounds * slots), width = units / tiles, more = units - tiles * width;
    if constexpr (SW) return width >= 2 ? go(eight, std::integral_constant<int, 4>{}, tiles, 0) : go(eight, std::integral_constant<int, 2>{}, tiles, more);
    else return width >= 4 ? go(eight, std::integral_constant<int, 4>{}, tiles, 0) : width == 3 ? go(eight, std::integral_constant<int, 3>{}, tiles, more)
              : width == 2 ? go(eight, std::integral_constant<int, 2>{}, tiles, more) : go(eight, std::integral_constant<int, 1>{}, tiles, more);
}

// What a many-rows launch needs of the workspace; 0: more than its offsets of 32 bits reach.
inline size_t wide_bytes(const Product& p, int rows) {
    const size_t pad = (size_t(rows) + 127) / 128 * 128, x = size_t((p.K + 127) / 128) * 256 * pad, n = size_t(p.N) * (p.epi == EPI_SWIGLU ? 2 : 1);
    return x >= size_t(1) << 31 || size_t(p.groups) * p.N * 2 >= size_t(1) << 31 ? 0 : x + pad * 4 + n * 4 + 16;
}

template <typename T, bool SW, int GS>
hipError_t choose(const Product& p, float* ws, size_t ws_bytes, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        const int64_t outputs = int64_t(p.N) * (SW ? 2 : 1);
        // Few rows: each four read the weights once more, which come from a cache then, but there is one launch and nothing between its workgroups.
        // rows / tiles, us: 4 rows, 4096 outputs of 4096 inputs 5.3 / 8.7, 16384 of 4096 10.8 / 13.0, 8192 of 8192 14.8 / 12.5, 28672 of 6144
        // 32.2 / 25.0; 8 rows, 6144 of 4096 8.6 / 10.2, 12288 of 4096 15.6 / 13.3; 32 rows, 2048 of 2048 6.2 / 10.0; 16 rows, 4096 of 4096 9.2 / 8.7;
        // 100 rows, gate and up of 2000, 256 11.5 / 7.3.  Inputs below 1024 cost as much: eight waves share them.
        if (p.M == 1 || (p.M <= 4 && p.K <= 4096) || (p.M + 3) / 4 * outputs * std::max(p.K, 1024) < int64_t(1) << 26) return rows<T, SW, GS>(p, st);
        // Many rows: the pass before the product costs some 8 us.  tiles / wide, us: 128 rows, 12288 outputs of 4096 inputs 36.6 / 28.4, 4096 of 14336
        // 33.5 / 34.4; 512 rows, 4096 of 4096 38.8 / 33.3, 1792 of 2048 22.5 / 17.7; 2048 rows, 4096 of 14336 354 / 245; up to 64 rows a tile's codes are
        // converted once.  Without room for the pass's activations in the workspace it is the tiles: 4096 rows, 4096 of 14336 705.
        const size_t need = wide_bytes(p, p.M);
        if (p.M > 64 && p.M * outputs >= 800000 && need && need <= ws_bytes) return wide<SW>(p, GS, ws, ws_bytes, st);
        return tiles<SW, GS>(p, ws, ws_bytes, st);
    }
    // Four rows at a time cost their share of the outputs and the inputs, tiles the inputs alone until the launch is full: rows / tiles, us: 732 rows, 3553 outputs,
    // 1320 inputs 206 / 37; 64, 4096, 4096 54 / 48; 256, gate and up of 688, 256 13.8 / 5.7; 128, 1024, 1024 8.4 / 13.2; 40, 2048, 2048 10.5 / 23.7.
    if constexpr (sizeof(T) == 4)
        if (p.M > 16 && int64_t((p.M + 3) / 4) * p.N * (SW ? 2 : 1) >= 50000) {
            hipLaunchKernelGGL((w4_f32_kernel<SW, GS>), dim3(unsigned((p.N + (SW ? 63 : 127)) / (SW ? 64 : 128)), unsigned((p.M + 31) / 32)), dim3(256), 0, st, p);
            return hipGetLastError();
        }
    return rows<T, SW, GS>(p, st);
}

template <typename T>
hipError_t product(const Product& p, int group, float* ws, size_t ws_bytes, hipStream_t st) {
    auto go = [&](auto sw) {
        constexpr bool SW = decltype(sw)::value;
        return group == 128 ? choose<T, SW, 128>(p, ws, ws_bytes, st) : group == 64 ? choose<T, SW, 64>(p, ws, ws_bytes, st) : choose<T, SW, 32>(p, ws, ws_bytes, st);
    };
    return p.epi == EPI_SWIGLU ? go(std::true_type{}) : go(std::false_type{});
}

template <typename T>
hipError_t pack(const T* w, unsigned char* codes, T* scales, T* values, int N, int K, int group, hipStream_t st) {
    const int groups = (K + group - 1) / group;
    const int rows = 256 / (group / 8);
    const dim3 grid(unsigned(std::min<int64_t>(int64_t((N + rows - 1) / rows) * groups, 1 << 22)));
    auto go = [&](auto gs) {
        hipLaunchKernelGGL((pack_w4_kernel<T, decltype(gs)::value>), grid, dim3(256), 0, st, w, codes, scales, values, N, K, (K + 31) / 32 * 16, groups);
        return hipGetLastError();
    };
    return group == 128 ? go(std::integral_constant<int, 128>{}) : group == 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 32>{});
}
}  // namespace

hipError_t launch_gemm_w4(int dtype, int epi, const void* a, const cake_w4& w, const cake_w4* w2, void* out, int M, float* ws, size_t ws_bytes, hipStream_t st) {
    const Product p = {a, (const unsigned char*)w.codes, w2 ? (const unsigned char*)w2->codes : nullptr, w.scales, w2 ? w2->scales : nullptr, out, nullptr,
                       M, w.n, w.k, (w.k + 31) / 32 * 16, (w.k + w.group - 1) / w.group, epi};
    return dtype == CAKE_F32 ? product<float>(p, w.group, ws, ws_bytes, st) : product<bf16_t>(p, w.group, ws, ws_bytes, st);
}

hipError_t launch_pack_w4(int dtype, const void* w, void* codes, void* scales, void* values, int N, int K, int group, hipStream_t st) {
    if (dtype == CAKE_F32) return pack((const float*)w, (unsigned char*)codes, (float*)scales, (float*)values, N, K, group, st);
    return pack((const bf16_t*)w, (unsigned char*)codes, (bf16_t*)scales, (bf16_t*)values, N, K, group, st);
}

}  // namespace cake
