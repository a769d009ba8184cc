// Products with 4-bit weights (layout: cake.h, cake_w4), and the packing of such weights.
//
// out[m][n] = sum over groups g of s[n][g] * (sum over the group's k of a[m][k] c[n][k]): the matrix cores multiply the activations by the
// codes, exact in bfloat16, a group's sum is kept apart and enters the result times its scale, one multiply-add.  Nothing is rounded
// on the way but float32 sums.
#include <algorithm>
#include <cmath>

#include "kernels.hpp"

namespace cake {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
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
__device__ __forceinline__ unsigned word(uint4 x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

template <typename T> struct Terms { static constexpr int N = 1; };
template <> struct Terms<float> { static constexpr int N = 3; };       // 24 bits in three bfloat16

struct Product {
    const void* a;
    const unsigned char *w, *w2;       // codes; w2: of up (SwiGLU)
    const void *s, *s2;                // scales
    void* out;
    int M, N, K, row_bytes, groups;
};

// A wave takes 16 NT outputs and every NW-th step of 128 inputs; a lane's 16 bytes of a row's codes are 32 inputs of it.  Groups of 128: the four
// lanes of a row multiply their first eight, second eight .. at once.  Shorter groups: the lanes exchange words first, so that
// a product's 32 inputs lie in one group.  The offset 24 of the codes: a group's sum begins with -24 times the sum of its
// activations, formed by a product with a constant operand that all outputs share.
template <typename T, int EPI, int MB, int NT, int GS, int NW>
__global__ void __launch_bounds__(64 * NW)
w4_rows_kernel(Product p) {
    constexpr int TERMS = Terms<T>::N, TWO = EPI == EPI_SWIGLU ? 2 : 1, NC = NT / TWO, PER = 128 / GS, MFMAS = 4 / PER;   // NC: tiles of outputs; PER: groups a step
    static_assert(NT % TWO == 0, "gate and up side by side");
    __shared__ float part[NW][MB][NT][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g4 = lane >> 4;
    const int n0 = blockIdx.x * (16 * NC), m0 = blockIdx.y * (16 * MB);
    const T* const a = (const T*)p.a;
    const int steps = (p.K + 127) / 128;
    const unsigned char* row[NT];
    const T* srow[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = min(n0 + 16 * (t % NC) + n16, p.N - 1);             // rows past the last: the last, not stored
        row[t] = (t < NC ? p.w : p.w2) + size_t(n) * p.row_bytes + g4 * 16;
        srow[t] = (const T*)(t < NC ? p.s : p.s2) + size_t(n) * p.groups;
    }
    const T* arow[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) arow[b] = a + size_t(min(m0 + 16 * b + n16, p.M - 1)) * p.K;
    f32x4 acc[MB][NT];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint4 minus24 = {0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u};
    const uint4 zero = {0, 0, 0, 0};

    for (int i = wave; i < steps; i += NW) {
        const int k0 = i * 128;
        uint4 w[NT];
        float s[NT][PER];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            w[t] = k0 + 32 * g4 < p.K ? *(const uint4*)(row[t] + i * 64) : zero;
#pragma unroll
            for (int g = 0; g < PER; ++g) s[t][g] = i * PER + g < p.groups ? float(srow[t][i * PER + g]) : 0.f;
        }
        bf16x8 x[MB][TERMS][4];
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + (GS == 128 ? 32 * g4 + 8 * j : 32 * j + 8 * g4);
                if constexpr (TERMS == 1) {
                    x[b][0][j] = in_order(k < p.K ? *(const uint4*)(arow[b] + k) : zero);
                } else {
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = k < p.K ? arow[b][k + (e >> 1) + 4 * (e & 1)] : 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int q = 0; q < TERMS; ++q) { x[b][q][j][e] = bf16_t(f[e]); f[e] -= float(x[b][q][j][e]); }
                }
            }
        if constexpr (GS < 128)
#pragma unroll
            for (int t = 0; t < NT; ++t) w[t] = transposed(w[t]);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            f32x4 begin[MB];
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                begin[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = g * MFMAS; j < (g + 1) * MFMAS; ++j)
#pragma unroll
                    for (int q = TERMS - 1; q >= 0; --q) begin[b] = mfma16(x[b][q][j], __builtin_bit_cast(bf16x8, minus24), begin[b]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f32x4 sum[MB];
#pragma unroll
                for (int j = g * MFMAS; j < (g + 1) * MFMAS; ++j) {
                    const bf16x8 c = codes8(word(w[t], j));
#pragma unroll
                    for (int b = 0; b < MB; ++b)
#pragma unroll
                        for (int q = TERMS - 1; q >= 0; --q) sum[b] = mfma16(x[b][q][j], c, j == g * MFMAS && q == TERMS - 1 ? begin[b] : sum[b]);
                }
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[b][t][v] = __builtin_fmaf(sum[b][v], s[t][g], acc[b][t][v]);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) part[wave][b][t][v][lane] = acc[b][t][v];
    __syncthreads();
    // the waves' parts in their order; D[4 g4 + v][n16]
    for (int i = threadIdx.x; i < MB * NC * 256; i += 64 * NW) {
        const int l = i & 63, v = i >> 6 & 3, t = (i >> 8) % NC, b = (i >> 8) / NC;
        const int m = m0 + 16 * b + 4 * (l >> 4) + v, n = n0 + 16 * t + (l & 15);
        float y = 0.f, y2 = 0.f;
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            y += part[q][b][t][v][l];
            if constexpr (TWO == 2) y2 += part[q][b][t + NC][v][l];
        }
        if (m >= p.M || n >= p.N) continue;
        const size_t at = size_t(m) * p.N + n;
        if constexpr (EPI == EPI_STORE_F32) ((float*)p.out)[at] = y;
        else if constexpr (EPI == EPI_RESIDUAL_F32) ((float*)p.out)[at] += y;
        else ((T*)p.out)[at] = T(y / (1.f + expf(-y)) * y2);
    }
}

// A lane takes eight weights of a row, the lanes of a group find its largest magnitude.  Bound by the bytes.
template <typename T, int GS>
__global__ void __launch_bounds__(256)
pack_w4_kernel(const T* __restrict__ w, unsigned char* __restrict__ codes, T* __restrict__ scales, T* __restrict__ values, int N, int K, int row_bytes, int groups) {
    constexpr int LANES = GS / 8;
    const int per_row = groups * LANES;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < int64_t(N) * per_row; i += int64_t(gridDim.x) * 256) {   // whole groups of lanes
        const int n = int(i / per_row), piece = int(i % per_row), k = piece * 8;
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
        if (piece % LANES == 0) scales[size_t(n) * groups + piece / LANES] = s;
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

template <typename T, int EPI, int GS>
hipError_t rows(const Product& p, hipStream_t st) {
    constexpr int NT = EPI == EPI_SWIGLU ? 2 : 1;
    auto go = [&](auto mb) {
        constexpr int MB = decltype(mb)::value;
        hipLaunchKernelGGL((w4_rows_kernel<T, EPI, MB, NT, GS, 4>), dim3(unsigned((p.N + 15) / 16), unsigned((p.M + 16 * MB - 1) / (16 * MB))), dim3(256), 0, st, p);
        return hipGetLastError();
    };
    if (p.M <= 16) return go(std::integral_constant<int, 1>{});
    return go(std::integral_constant<int, 2>{});
}

template <typename T, int EPI>
hipError_t by_group(const Product& p, int group, hipStream_t st) {
    return group == 128 ? rows<T, EPI, 128>(p, st) : group == 64 ? rows<T, EPI, 64>(p, st) : rows<T, EPI, 32>(p, st);
}

template <typename T>
hipError_t by_form(int epi, const Product& p, int group, hipStream_t st) {
    return epi == EPI_STORE_F32 ? by_group<T, EPI_STORE_F32>(p, group, st) : epi == EPI_RESIDUAL_F32 ? by_group<T, EPI_RESIDUAL_F32>(p, group, st)
                                                                                                     : by_group<T, EPI_SWIGLU>(p, group, st);
}

template <typename T>
hipError_t pack(const T* w, unsigned char* codes, T* scales, T* values, int N, int K, int group, hipStream_t st) {
    const int groups = (K + group - 1) / group;
    const dim3 grid(unsigned(std::min<int64_t>((int64_t(N) * groups * (group / 8) + 255) / 256, 1 << 22)));
    auto go = [&](auto gs) {
        hipLaunchKernelGGL((pack_w4_kernel<T, decltype(gs)::value>), grid, dim3(256), 0, st, w, codes, scales, values, N, K, (K + 31) / 32 * 16, groups);
        return hipGetLastError();
    };
    return group == 128 ? go(std::integral_constant<int, 128>{}) : group == 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 32>{});
}
}  // namespace

hipError_t launch_gemm_w4(int dtype, int epi, const void* a, const cake_w4& w, const cake_w4* w2, void* out, int M, hipStream_t st) {
    const Product p = {a, (const unsigned char*)w.codes, w2 ? (const unsigned char*)w2->codes : nullptr, w.scales, w2 ? w2->scales : nullptr, out, M, w.n, w.k,
                       (w.k + 31) / 32 * 16, (w.k + w.group - 1) / w.group};
    return dtype == CAKE_F32 ? by_form<float>(epi, p, w.group, st) : by_form<bf16_t>(epi, p, w.group, st);
}

hipError_t launch_pack_w4(int dtype, const void* w, void* codes, void* scales, void* values, int N, int K, int group, hipStream_t st) {
    if (dtype == CAKE_F32) return pack((const float*)w, (unsigned char*)codes, (float*)scales, (float*)values, N, K, group, st);
    return pack((const bf16_t*)w, (unsigned char*)codes, (bf16_t*)scales, (bf16_t*)values, N, K, group, st);
}

}  // namespace cake
