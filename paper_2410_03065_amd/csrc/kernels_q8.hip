// A ragged batch over an 8-bit paged cache (layout: cake.h, cake_q8_batch): appending rotated keys and values, and
// attention that reads the codes.
//
// Key j of a KV head stands for the vector c_j * s_j: int8 codes c_j and the float32 scale s_j of the block of tokens that
// it lies in.  A score is therefore (q . c_j) * s_j and an output sum_j (p_j s'_j) c'_j: the products run on the codes as they
// are, exact in bfloat16 (eight bits), and a scale is one factor per score.  No dequantised copy of the cache exists anywhere.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>

#include "kernels.hpp"

namespace cake {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// v_mfma_f32_16x16x32_bf16, D[16x16] += A[16x32] * B[32x16]: lane l supplies A[l%16][8*(l/16) .. +7] and
// B[8*(l/16) .. +7][l%16], and holds D[4*(l/16) + v][l%16] in accumulator register v (0..3).
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ unsigned pack_hi(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }
// byte j of w as a signed number: one instruction, and exact in bfloat16, so that its upper half is the bfloat16
__device__ __forceinline__ float code(unsigned w, int j) { return float((signed char)(w >> (8 * j))); }
__device__ __forceinline__ bf16x8 codes8(unsigned lo, unsigned hi) {
    const uint4 r = {pack_hi(code(lo, 0), code(lo, 1)), pack_hi(code(lo, 2), code(lo, 3)), pack_hi(code(hi, 0), code(hi, 1)), pack_hi(code(hi, 2), code(hi, 3))};
    return __builtin_bit_cast(bf16x8, r);
}
// Maximum / sum over the four lanes that share l % 16.
__device__ __forceinline__ float max4(float y) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Maximum over the 16 lanes of a row.
__device__ __forceinline__ float max16(float y) {
    y = fmaxf(y, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x121, 0xf, 0xf, false)));   // row_ror:1, 2, 4, 8
    y = fmaxf(y, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x122, 0xf, 0xf, false)));
    y = fmaxf(y, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x124, 0xf, 0xf, false)));
    return fmaxf(y, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x128, 0xf, 0xf, false)));
}
__device__ __forceinline__ float sum4(float y) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The batch's arrays are read with uniform indexes and never written by a kernel: through the scalar cache, so that a read
// waits for no vector load before it.
__device__ __forceinline__ int uniform(const int32_t* p, size_t i) { return ((const __attribute__((address_space(4))) int32_t*)p)[i]; }

// A sequence of the batch.  What the device arrays say is not trusted: rows stay inside [0, n_rows), and a length that the
// block table cannot hold (over) is never followed.
struct Seq { int row0, rows, len; bool over; };
__device__ __forceinline__ Seq sequence(const Q8View& v, int s) {
    Seq q;
    q.row0 = min(max(uniform(v.row_begin, s), 0), v.n_rows);
    q.rows = min(max(uniform(v.row_begin, s + 1), q.row0), v.n_rows) - q.row0;
    q.len = min(max(uniform(v.seq_len, s), 0), Q8_MOST_TOKENS);
    q.over = q.len > v.pages_per_seq * v.page_tokens;
    return q;
}

template <typename T> __device__ __forceinline__ T to_elem(float x);
template <> __device__ __forceinline__ float to_elem<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t to_elem<bf16_t>(float x) { return bf16_t(x); }

template <typename T, int N> struct Vec { typedef T type __attribute__((__vector_size__(N * sizeof(T)))); };

// ===================================================================================== append
// Cosine and sine of x >= 0 (radians) to some units of 2^-53: x less the nearest multiple of pi / 2, which is subtracted in three
// parts of 53 bits (the quotient has at most 30), then Taylor polynomials on |r| <= pi / 4, whose first terms left out are
// 0.785^17 / 17! = 5e-17 and 0.785^18 / 18! = 2e-18.
__device__ __forceinline__ void turn(double x, double* cosine, double* sine) {
    const double k = rint(x * 0.63661977236758134308);
    double r = fma(-k, 1.5707963267948966, x);
    r = fma(-k, 6.123233995736766e-17, r);
    r = fma(-k, -1.4973849048591833e-33, r);
    const double z = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = fma(s, z, 1.0 / 6227020800.0); c = fma(c, z, -1.0 / 87178291200.0);
    s = fma(s, z, -1.0 / 39916800.0);  c = fma(c, z, 1.0 / 479001600.0);
    s = fma(s, z, 1.0 / 362880.0);     c = fma(c, z, -1.0 / 3628800.0);
    s = fma(s, z, -1.0 / 5040.0);      c = fma(c, z, 1.0 / 40320.0);
    s = fma(s, z, 1.0 / 120.0);        c = fma(c, z, -1.0 / 720.0);
    s = fma(s, z, -1.0 / 6.0);         c = fma(c, z, 1.0 / 24.0);
    s = fma(s * z, r, r);              c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const int quarter = int(k) & 3;
    const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    *cosine = quarter == 1 || quarter == 2 ? -a : a;
    *sine = quarter & 2 ? -b : b;
}

// How a head's elements lie on the 16 lanes that hold it: side by side (adjacent pairs; halves of part of the head, whose
// partners are read again), or as many of each half where all of the head turns in halves, partners in one lane.
enum RopeMode { ROPE_ADJACENT, ROPE_HALVES, ROPE_HALVES_PART };

// Two kinds of workgroups.  Rows: eight tokens of a sequence and some of the heads, sixteen heads' rows at a time, four more on
// their way; with a scale per token that is all.  Blocks, where tokens share scales: 64 positions (whole blocks, aligned, so no
// two workgroups write one) of one KV head, whose keys and values stay in registers between the largest magnitude and the codes.
// They take longest and come first in the grid (last: 49 us, first: 38).
// Bound by the bytes: 4 read per element, 1 or 2 written; 2447 tokens of 64 / 8 heads of 128, a scale for 64: 38 us, 4.1 TB/s.  The rotation runs in 64 bits, full rate on this chip: at position 60000
// a float32 angle is off by 4e-3, and the codes that follow are whole numbers, which with the rotated value correctly rounded to
// float32 hardly depend on how cosine and sine were come by.
template <typename T, int HD, int MODE>
__global__ void __launch_bounds__(256)
append_q8_kernel(const float* __restrict__ qkv, T* __restrict__ q, T* __restrict__ values, Q8View v, cake_rope rope, int n_q, int row_tiles, int chunks,
                 int block_groups, int block_tiles) {
    constexpr int E = HD / 16, P = MODE == ROPE_HALVES ? E / 2 : E, S = MODE == ROPE_HALVES ? HD / 2 : 0;   // elements a lane, in a piece; pieces apart
    constexpr int TOKENS = 8, AT_ONCE = 4, HELD = 8;
    typedef typename Vec<float, P < 4 ? P : 4>::type Piece;
    constexpr int PW = P < 4 ? P : 4;
    __shared__ double2 cs[TOKENS * (HD / 2)];       // rows: cosine and sine of the tokens' pairs
    __shared__ unsigned amax[2][64];                // blocks: the largest magnitude, then the scale
    __shared__ float ratio[2];                      // what the codes of the first block's older tokens are multiplied by
    const int tid = threadIdx.x, group = tid >> 4, lane = tid & 15, e0 = lane * P;
    const int half = rope.rotary_dim / 2, block = 1 << v.scale_shift, all_heads = n_q + 2 * v.n_kv;
    const int cap = v.pages_per_seq * v.page_tokens;
    auto at = [&](int e) { return e < P ? e0 + e : e0 + S + e - P; };     // the place of a lane's element in its head

    auto read = [&](const float* p, float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; e += PW) {
            const Piece w = *(const Piece*)(p + at(e));
#pragma unroll
            for (int k = 0; k < PW; ++k) x[e + k] = w[k];
        }
    };
    // rotated in 64 bits, rounded to float32; pair(i): cosine and sine, p: the row (for partners in other lanes)
    auto rotate = [&](float (&x)[E], auto pair, const float* p) {
        if constexpr (MODE == ROPE_HALVES) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const double2 z = pair(e0 + e);
                const double a = x[e], b = x[e + P];
                x[e] = float(a * z.x - b * z.y);
                x[e + P] = float(a * z.y + b * z.x);
            }
        } else if constexpr (MODE == ROPE_ADJACENT) {
#pragma unroll
            for (int e = 0; e < E; e += 2)
                if (e0 + e < rope.rotary_dim) {
                    const double2 z = pair((e0 + e) / 2);
                    const double a = x[e], b = x[e + 1];
                    x[e] = float(a * z.x - b * z.y);
                    x[e + 1] = float(a * z.y + b * z.x);
                }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e0 + e < rope.rotary_dim) {
                    const bool first = e0 + e < half;
                    const double2 z = pair(first ? e0 + e : e0 + e - half);
                    const double y = p[first ? e0 + e + half : e0 + e - half];
                    x[e] = float(first ? double(x[e]) * z.x - y * z.y : double(x[e]) * z.x + y * z.y);
                }
        }
    };
    auto store = [&](T* d, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; e += P) {
            typename Vec<T, P>::type o;
#pragma unroll
            for (int k = 0; k < P; ++k) o[k] = to_elem<T>(x[e + k]);
            *(typename Vec<T, P>::type*)(d + at(e)) = o;
        }
    };
    // the row's largest magnitude, as bits: they order like the numbers, and infinities and NaN come out on top
    auto largest = [&](const float (&x)[E]) {
        unsigned m = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
        m = max(m, unsigned(__builtin_amdgcn_update_dpp(0, int(m), 0x121, 0xf, 0xf, false)));   // row_ror:1, 2, 4, 8
        m = max(m, unsigned(__builtin_amdgcn_update_dpp(0, int(m), 0x122, 0xf, 0xf, false)));
        m = max(m, unsigned(__builtin_amdgcn_update_dpp(0, int(m), 0x124, 0xf, 0xf, false)));
        return max(m, unsigned(__builtin_amdgcn_update_dpp(0, int(m), 0x128, 0xf, 0xf, false)));
    };
    auto scale_of = [](unsigned m) { return m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(m) / 127.0f; };
    auto page_of = [&](int s, int pos) -> unsigned char* {   // null where nothing can be written
        if (pos >= cap) return nullptr;
        const int phys = v.table[size_t(s) * v.pages_per_seq + pos / v.page_tokens];
        return phys < 0 || phys >= v.n_phys ? nullptr : v.base + size_t(phys) * v.page_bytes;
    };
    // a token's codes of one head (which: 0 key, 1 value) into its page, and what they stand for
    auto put = [&](const float (&x)[E], int which, int g, int pos, size_t row, float scale, unsigned char* page) {
        float c[E];
        unsigned w[E / P] = {}, wide[E / P] = {};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            c[e] = scale > 0.f ? fminf(fmaxf(rintf(x[e] / scale), -127.f), 127.f) : 0.f;
            const int k = e % P;
            (k < 4 ? w : wide)[e / P] |= (unsigned(int(c[e])) & 255u) << (8 * (k & 3));
        }
        if (page) {
            const int off = pos % v.page_tokens;
            unsigned char* half_page = page + which * v.half_bytes;
            unsigned char* d = half_page + (size_t(g) * v.page_tokens + off) * HD;
#pragma unroll
            for (int k = 0; k < E / P; ++k) {
                if constexpr (P == 8) *(uint2*)(d + at(k * P)) = uint2{w[k], wide[k]};
                else if constexpr (P == 4) *(unsigned*)(d + at(k * P)) = w[k];
                else *(unsigned short*)(d + at(k * P)) = (unsigned short)w[k];
            }
            if (block == 1 && lane == 0) ((float*)(half_page + v.scales_off))[size_t(g) * v.page_tokens + off] = scale;
        }
        if (values) {
#pragma unroll
            for (int e = 0; e < E; ++e) c[e] = page ? c[e] * scale : __uint_as_float(0x7fc00000u);
            store(values + (row * 2 * v.n_kv + which * v.n_kv + g) * HD, c);
        }
    };
    auto pair_at = [&](int pos, int i) {
        double2 z;
        turn(double(pos) * rope.freq[i], &z.x, &z.y);
        return double2{z.x * rope.magnitude, z.y * rope.magnitude};
    };

    if (int(blockIdx.x) >= block_groups) {
        // ---- rows
        int b = int(blockIdx.x) - block_groups;
        const int chunk = b % chunks; b /= chunks;
        const int t0 = b % row_tiles, s = b / row_tiles;
        const Seq seq = sequence(v, s);
        const int p0 = seq.len - seq.rows, p_new = max(p0, 0);   // rows in excess of the sequence's tokens stand for no token
        const int heads = block == 1 ? all_heads : n_q;
        const int h0 = int(int64_t(heads) * chunk / chunks), nh = int(int64_t(heads) * (chunk + 1) / chunks) - h0;
        for (int t = t0; p_new + t * TOKENS < seq.len; t += row_tiles) {
            const int lo = p_new + t * TOKENS, n = min(TOKENS, seq.len - lo), items = n * nh;
            if (t != t0) __syncthreads();
            if (h0 < n_q + v.n_kv)
                for (int i = tid; i < n * half; i += 256) {
                    const int tok = i / half, f = i - tok * half;
                    cs[tok * (HD / 2) + f] = pair_at(lo + tok, f);
                }
            __syncthreads();
            for (int i0 = group; i0 < items; i0 += 16 * AT_ONCE) {
                float x[AT_ONCE][E];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int i = min(i0 + 16 * k, items - 1), tok = i / nh, h = h0 + i - tok * nh;
                    read(qkv + (size_t(seq.row0 + lo - p0 + tok) * all_heads + h) * HD, x[k]);
                }
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int i = i0 + 16 * k;
                    if (i >= items) break;
                    const int tok = i / nh, h = h0 + i - tok * nh, pos = lo + tok;
                    const size_t row = seq.row0 + lo - p0 + tok;
                    if (h < n_q + v.n_kv) rotate(x[k], [&](int f) { return cs[tok * (HD / 2) + f]; }, qkv + (row * all_heads + h) * HD);
                    if (h < n_q) store(q + (size_t(h) * v.n_rows + row) * HD, x[k]);
                    else put(x[k], h >= n_q + v.n_kv, (h - n_q) % v.n_kv, pos, row, scale_of(largest(x[k])), page_of(s, pos));
                }
            }
        }
        return;
    }
    // ---- blocks
    int b = blockIdx.x;
    const int g = b % v.n_kv; b /= v.n_kv;
    const int t0 = b % block_tiles, s = b / block_tiles;
    const Seq seq = sequence(v, s);
    const int p0 = seq.len - seq.rows, p_new = max(p0, 0), first = p_new / 64 * 64, blocks = 64 >> v.scale_shift;
    for (int t = t0; first + t * 64 < seq.len; t += block_tiles) {
        const int base = first + t * 64, lo = max(base, p_new), n = min(base + 64, seq.len) - lo;
        if (n <= 0) return;
        if (t != t0) __syncthreads();
        float x[HELD][E];
        auto row_of = [&](int i) { return size_t(seq.row0 + lo - p0 + (i >> 1)); };
        auto from = [&](int i) { return qkv + (row_of(i) * all_heads + n_q + (i & 1) * v.n_kv + g) * HD; };
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (group + 16 * k < 2 * n) read(from(group + 16 * k), x[k]);
        if (tid < 128) amax[tid >> 6][tid & 63] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int i = group + 16 * k;
            if (i >= 2 * n) break;
            if (!(i & 1)) rotate(x[k], [&](int f) { return pair_at(lo + (i >> 1), f); }, from(i));
            const unsigned m = largest(x[k]);
            if (lane == 0) atomicMax(&amax[i & 1][(lo + (i >> 1) - base) >> v.scale_shift], m);
        }
        __syncthreads();
        unsigned char* const page = page_of(s, base);               // 64 positions lie in one page
        if (tid < 2 * blocks) {
            const int which = tid & 1, k = tid >> 1, start = base + (k << v.scale_shift);
            const unsigned m = amax[which][k];
            float scale = scale_of(m);
            if (page && start < lo + n && start + block > lo) {
                float* where = (float*)(page + which * v.half_bytes + v.scales_off) + ((size_t(g) * v.page_tokens + start % v.page_tokens) >> v.scale_shift);
                if (start < lo) {                                    // the block holds older tokens
                    const float old = *where;
                    if (!(old <= scale)) scale = old;                 // also where either is NaN
                    if (m >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);
                    ratio[which] = scale > 0.f ? old / scale : 1.f;
                }
                *where = scale;
            }
            amax[which][k] = __float_as_uint(scale);
        }
        __syncthreads();
        const int start = lo / block * block, words = (lo - start) * (HD / 4);   // the older tokens of the first block
        for (int i = tid; page && i < 2 * words; i += 256) {
            const int which = i >= words, j = which ? i - words : i;
            const float r = ratio[which];
            if (!(r < 1.f)) continue;
            unsigned* d = (unsigned*)(page + which * v.half_bytes + (size_t(g) * v.page_tokens + start % v.page_tokens) * HD) + j;
            const unsigned old = *d;
            unsigned w = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) w |= (unsigned(int(fminf(fmaxf(rintf(code(old, k) * r), -127.f), 127.f))) & 255u) << (8 * k);
            *d = w;
        }
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int i = group + 16 * k;
            if (i >= 2 * n) break;
            const int pos = lo + (i >> 1);
            put(x[k], i & 1, g, pos, row_of(i), __uint_as_float(amax[i & 1][(pos - base) >> v.scale_shift]), page);
        }
    }
}

// ===================================================================================== attention
// The keys that some row of a tile of rows sees, in steps of W: the steps of the first tokens that stay visible, then from
// the window's (step number i stands for step at(i)).
template <int W> struct KeySteps {
    int sink_steps, first, n;
    __device__ __forceinline__ int at(int i) const { return i < sink_steps ? i : first + i - sink_steps; }
};
// Is a key seen by one of the rows at positions lo .. hi?  (window: Q8_MOST_TOKENS where there is none.)
__device__ __forceinline__ bool visible(int key, int lo, int hi, int window, int sinks) { return (key <= hi) & ((key > lo - window) | (key < sinks)); }
template <int W> __device__ __forceinline__ KeySteps<W> key_steps(int pos_lo, int pos_hi, int window, int sinks) {
    KeySteps<W> k = {0, 0, 0};
    if (pos_hi < 0) return k;
    if (pos_lo - window + 1 > 0) {
        k.first = (pos_lo - window + 1) / W;
        k.sink_steps = (min(sinks, pos_lo - window + 1) + W - 1) / W;
        if (k.sink_steps >= k.first) k.first = k.sink_steps = 0;
    }
    k.n = k.sink_steps + pos_hi / W + 1 - k.first;
    return k;
}

// Few rows.  A tile is NB x 16 rows (token, query head of the group) of one sequence and KV head; a workgroup takes a range of
// its key steps, its four (eight) waves every fourth (eighth) step each, straight from memory into registers.  Scores are formed transposed,
// S^T[key][row] = K Q^T, so that a lane holds four keys of one row per block of 16 and the weights are the second product's
// operand as they are: O^T[hd][row] += V^T W^T, where the slots of a product are dealt to keys as the scores lie (slot
// 8g + t: key 4g + t, from t = 4 key 16 + 4g + t - 4).  A lane reads 8 (4) neighbouring elements of eight keys' values and
// its conversions pick the bytes, so nothing is transposed.  Bound by the cache's bytes; per byte 1.5 vector instructions.
// Weights go to the product as two bfloat16 values each (16 bits; float32 models: three, all 24, as the queries): at this
// size the matrix cores are idle, and a single bfloat16 would double the output's rounding error.
// Measured: 64 sequences of 500 to 8191 keys, 8 KV heads of 128: 126 us, 4.7 TB/s; 24 of 4100 visible keys, 32 KV heads: 147 us, 5.5 TB/s.
template <typename T> struct Terms { static constexpr int Q = 1, W = 2; };
template <> struct Terms<float> { static constexpr int Q = 3, W = 3; };

template <typename T, int HD, int NB, int NS, int NW>
__global__ void __launch_bounds__(64 * NW, NW == 8 || NB == 2 || Terms<T>::Q == 3 ? 2 : HD == 128 ? 3 : 4)
attention_q8_kernel(const T* __restrict__ q, T* __restrict__ out, float* __restrict__ part, Q8View v, int n_q, int window, int sinks,
                    float scale_log2, int chunk, int splits, int tiles) {
    constexpr int TQ = Terms<T>::Q, TW = Terms<T>::W;
    constexpr int QC = HD / 32, CW = HD / 16, KB = HD / 4;   // products per 16 keys; value columns and key bytes per lane
    __shared__ float s_acc[4][16][HD + 4], s_ml[4][16][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g4 = lane >> 4;
    unsigned b = blockIdx.x;
    const int g = b % v.n_kv; b /= v.n_kv;
    const int split = b % splits; b /= splits;
    const int tile0 = b % tiles, s = b / tiles;
    const int G = n_q / v.n_kv;
    const Seq seq = sequence(v, s);
    const int n = seq.rows * G, p0 = seq.len - seq.rows;

    for (int tile = tile0; tile * (16 * NB) < n; tile += tiles) {
        if (tile != tile0) __syncthreads();
        const int i0 = tile * (16 * NB), i1 = min(i0 + 16 * NB, n) - 1;
        const int pos_lo = p0 + i0 / G, pos_hi = p0 + i1 / G;
        KeySteps<32> ks = key_steps<32>(pos_lo, pos_hi, window, sinks);
        if (seq.over) ks.n = 0;
        const int c0 = split * chunk, c1 = split == splits - 1 ? ks.n : min(ks.n, c0 + chunk);
        // this lane's row of each block of 16: the query (B operand), its position
        bf16x8 qf[NB][TQ][QC];
        int pos[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            const int i = i0 + 16 * r + n16;
            pos[r] = i < n ? p0 + i / G : -1;
            const T* p = q + (size_t(g * G + (i < n ? i % G : 0)) * v.n_rows + seq.row0 + (i < n ? i / G : 0)) * HD + g4 * KB;
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                if constexpr (TQ == 1) {
                    qf[r][0][c] = *(const bf16x8*)(p + 8 * c);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float x = p[8 * c + e];
#pragma unroll
                        for (int t = 0; t < TQ; ++t) { qf[r][t][c][e] = bf16_t(x); x -= float(qf[r][t][c][e]); }
                    }
                }
            }
        }
        f32x4 acc[NB][CW];
        float m[NB], l[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            m[r] = -FLT_MAX; l[r] = 0.f;
#pragma unroll
            for (int j = 0; j < CW; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // One step's raw bytes: the next step's keys are asked for when these have been multiplied, its values likewise, so a
        // wave has a step in flight while it works, in half the registers of two sets (and twice the waves).
        uint4 kr[2][KB / 16];
        uint2 vr[8];
        float ksc[2][NS], vsc[2][NS];
        const unsigned char* page = nullptr;       // the page of the step asked for last, and its first key's place there
        int off = 0, phys = -1;
        auto look_up = [&](int i) {                // a step's physical page, asked for a step ahead of its keys
            const int key0 = ks.at(i) * 32, pg = key0 / v.page_tokens;
            off = key0 - pg * v.page_tokens;
            phys = uniform(v.table, size_t(s) * v.pages_per_seq + pg);
        };
        auto scales = [&](float (&d)[2][NS], const unsigned char* from) {
            const float* p = (const float*)from;
            const int at = g * v.page_tokens + off + 4 * g4;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (NS == 4) *(float4*)d[h] = *(const float4*)(p + at + 16 * h);
                else d[h][0] = p[(at + 16 * h) >> v.scale_shift];
            }
        };
        bool bad = false;                          // keys of a page outside the pool: whoever sees them gets NaN
        auto load_keys = [&] {
            bad = phys < 0 || phys >= v.n_phys;
            page = v.base + size_t(bad ? 0 : phys) * v.page_bytes;
            const unsigned char* kc = page + (size_t(g) * v.page_tokens + off) * HD;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < KB / 16; ++c) kr[h][c] = *(const uint4*)(kc + (16 * h + n16) * HD + g4 * KB + 16 * c);
            scales(ksc, page + v.scales_off);
        };
        auto load_values = [&] {
            const unsigned char* vc = page + v.half_bytes + (size_t(g) * v.page_tokens + off) * HD;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const unsigned char* p = vc + ((t < 4 ? 0 : 12) + 4 * g4 + t) * HD + n16 * CW;
                if constexpr (CW == 8) vr[t] = *(const uint2*)p;
                else vr[t].x = *(const unsigned*)p;
            }
            scales(vsc, page + v.half_bytes + v.scales_off);
        };
        int i = c0 + wave;
        if (i < c1) { look_up(i); load_keys(); load_values(); }
        for (; i < c1; i += NW) {
            const int key0 = ks.at(i) * 32;
            const bool more = i + NW < c1, was_bad = bad;
            if (more) look_up(i + NW);
            const bool edge = key0 + 31 > pos_lo || (key0 <= pos_hi - window && key0 + 31 >= sinks);
            f32x4 sc[NB][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int r = 0; r < NB; ++r) sc[r][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    const uint4 w = kr[h][c / 2];
                    const bf16x8 kf = c & 1 ? codes8(w.z, w.w) : codes8(w.x, w.y);
#pragma unroll
                    for (int t = TQ - 1; t >= 0; --t)
#pragma unroll
                        for (int r = 0; r < NB; ++r) sc[r][h] = mfma16(kf, qf[r][t][c], sc[r][h]);
                }
#pragma unroll
                for (int r = 0; r < NB; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[r][h][e] *= (was_bad ? __uint_as_float(0x7fc00000u) : ksc[h][e % NS]) * scale_log2;
            }
            if (more) load_keys();
            bf16x8 wf[NB][TW];
#pragma unroll
            for (int r = 0; r < NB; ++r) {
                if (edge) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sc[r][h][e] = visible(key0 + 16 * h + 4 * g4 + e, pos[r], pos[r], window, sinks) ? sc[r][h][e] : -INFINITY;
                        }
                }
                float top = m[r];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[r][h][e]);
                top = max4(top);
                if (__builtin_amdgcn_ballot_w64(top > m[r])) {
                    const float f = __builtin_amdgcn_exp2f(m[r] - top);
                    l[r] *= f;
#pragma unroll
                    for (int j = 0; j < CW; ++j) acc[r][j] *= f;
                    m[r] = top;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(sc[r][h][e] - top);
                        l[r] += p;
                        // a hidden key's scale may be anything: memory behind the last token
                        float w = edge && sc[r][h][e] == -INFINITY ? 0.f : p * vsc[h][e % NS];
#pragma unroll
                        for (int t = 0; t < TW; ++t) { wf[r][t][4 * h + e] = bf16_t(w); w -= float(wf[r][t][4 * h + e]); }
                    }
            }
#pragma unroll
            for (int j = 0; j < CW; ++j) {
                uint4 a;
                auto col = [&](int t) { return code(j < 4 ? vr[t].x : vr[t].y, j & 3); };
                a.x = pack_hi(col(0), col(1)); a.y = pack_hi(col(2), col(3)); a.z = pack_hi(col(4), col(5)); a.w = pack_hi(col(6), col(7));
                const bf16x8 vf = __builtin_bit_cast(bf16x8, a);
#pragma unroll
                for (int r = 0; r < NB; ++r)
#pragma unroll
                    for (int t = TW - 1; t >= 0; --t) acc[r][j] = mfma16(vf, wf[r][t], acc[r][j]);
            }
            if (more) load_values();
        }
        // the waves' parts, added up in their order: of eight the upper four's first, each to the wave four below
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            if (r) __syncthreads();
            float lt = sum4(l[r]);
            auto leave = [&](int w) {
                if (g4 == 0) { s_ml[w][n16][0] = m[r]; s_ml[w][n16][1] = lt; }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < CW; j += 4)
                        *(float4*)&s_acc[w][n16][(4 * g4 + e) * CW + j] = make_float4(acc[r][j][e], acc[r][j + 1][e], acc[r][j + 2][e], acc[r][j + 3][e]);
            };
            if constexpr (NW == 8) {
                if (wave >= 4) leave(wave - 4);
                __syncthreads();
                if (wave < 4) {
                    const float other = s_ml[wave][n16][0], top = fmaxf(m[r], other);
                    const float f = __builtin_amdgcn_exp2f(m[r] - top), h = __builtin_amdgcn_exp2f(other - top);
                    lt = lt * f + s_ml[wave][n16][1] * h;
                    m[r] = top;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < CW; ++j) acc[r][j][e] = acc[r][j][e] * f + s_acc[wave][n16][(4 * g4 + e) * CW + j] * h;
                }
                __syncthreads();
            }
            if (wave < 4) leave(wave);
            __syncthreads();
            const int row = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * CW, idx = i0 + 16 * r + row;
            if (row < 16 && idx < n) {
                float mt = s_ml[0][row][0];
#pragma unroll
                for (int w = 1; w < 4; ++w) mt = fmaxf(mt, s_ml[w][row][0]);
                float sum = 0.f, o[CW] = {};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float f = __builtin_amdgcn_exp2f(s_ml[w][row][0] - mt);
                    sum += s_ml[w][row][1] * f;
#pragma unroll
                    for (int e = 0; e < CW; ++e) o[e] += s_acc[w][row][e0 + e] * f;
                }
                if (seq.over) sum = __uint_as_float(0x7fc00000u);
                const int trow = seq.row0 + idx / G, head = g * G + idx % G;
                if (splits == 1) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    T* d = out + (size_t(trow) * n_q + head) * HD + e0;
                    typename Vec<T, CW>::type ov;
#pragma unroll
                    for (int e = 0; e < CW; ++e) ov[e] = to_elem<T>(o[e] * inv);
                    *(typename Vec<T, CW>::type*)d = ov;
                } else {
                    float* d = part + ((size_t(trow) * n_q + head) * splits + split) * (HD + 4);
                    if (sum != 0.f)
#pragma unroll
                        for (int e = 0; e < CW; e += 4) *(float4*)(d + e0 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    if (e0 == 0) { d[HD] = mt; d[HD + 1] = sum; }
                }
            }
        }
    }
}

// Many rows.  A workgroup takes 32 rows (token, query head of the group) per wave and tiles of 64 keys, whose codes it converts
// once for all of them on the way into LDS: keys as bfloat16 [key][hd], values as half precision [hd][key slot], both exact.
// A weight is exp2(score - m), times its value's scale / 2^E in half precision.  m follows a row's maximum only when a weight
// would pass 2^11, so the outputs are hardly ever rescaled and rows exchange nothing between lanes on the way.  E is the
// exponent of the tile's largest scale, kept while it moves by less than 8 times; the outputs are in units of 2^E and move with it.
// So eleven bits are kept whatever the range of the scales (a single bfloat16, eight bits, would double the output's rounding
// error), and the largest product stays under 2^15.  A scale that is not finite is left out of the products: it is a bit in the
// tile's mask, rows that see its key get a NaN sum, and the others nothing.
// Scores transposed, key slots and the operands' order as above.
// The waves form two halves that alternate: while one multiplies, the other weighs its scores and asks for what comes next, so loads are
// a phase older than their use; codes are converted half-way through the products, and operands are read from LDS four products ahead, the
// first of them before the barrier.
// Bound by the vector instructions beside the products: a score takes 5 and an exponential (four times the issue of one), a
// code 1.5 over the workgroup's rows.  1024 rows of 32 heads after 15360 keys, 8 KV heads of 128: 330 to 390 us with the clock, 0.7 to
// 0.8 PFLOP/s; with products, weights and the rest each left alone, 131, 81 and 195.
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
__device__ __forceinline__ f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ unsigned pack_half(float a, float b) { return __builtin_bit_cast(unsigned, f16x2{_Float16(a), _Float16(b)}); }

// Of whole numbers up to 127, which need no rounding: one instruction a pair.
__device__ __forceinline__ unsigned pack_code(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(a, b)); }

// A barrier that waits for LDS alone: the next tiles' loads from memory stay in flight across it.
__device__ __forceinline__ void phase_end() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

constexpr float W_TOP = 11.f, W_FIRST = 6.f;      // largest exponent of a weight; where a row's maximum is put

template <int HD> struct RowsLds {
    static constexpr int K_BYTES = 64 * HD * 2, TILE = 2 * K_BYTES;
    static constexpr int KSC = 2 * TILE, VSC = KSC + 3 * 64 * 4, INFO = VSC + 3 * 64 * 4, BYTES = INFO + 3 * 16;
};

template <int HD, int NWV, int NS>
__global__ void __launch_bounds__(64 * NWV, 2)
attention_q8_rows_kernel(const bf16_t* __restrict__ q, bf16_t* __restrict__ out, float* __restrict__ part, Q8View v, int n_q, int window, int sinks,
                         float scale_log2, int chunk, int splits, int tiles) {
    constexpr int ROWS = 32 * NWV, HALF = 32 * NWV, CPT = 64 * HD / HALF, VC = CPT / 8;   // threads that stage one half; codes and columns of each
    constexpr int QC = HD / 32, HB = HD / 16;
    static_assert(VC == 4 || VC == 8, "values are loaded in pieces of four or eight codes");
    typedef RowsLds<HD> L;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g4 = lane >> 4;
    unsigned b = blockIdx.x;
    const int g = b % v.n_kv; b /= v.n_kv;
    const int split = b % splits; b /= splits;
    const int tile0 = b % tiles, s = b / tiles;
    const int G = n_q / v.n_kv;
    const Seq seq = sequence(v, s);
    const int n = seq.rows * G, p0 = seq.len - seq.rows;
    const bool keys_half = wave < NWV / 2;
    const int st = keys_half ? tid : tid - HALF;              // thread of its half
    const int k_key = st / (HD / CPT), k_at = st % (HD / CPT) * CPT;                          // keys: CPT codes of one key
    const int v_oct = st & 7, v_col = (st >> 3) * VC;                                         // values: VC columns of eight keys
    const int v_key = (v_oct >> 2) * 32 + (v_oct & 3) * 4;                                  // ... v_key + 0..3 and + 16..19
    // Pieces of 16 bytes in LDS rows: a key's piece p at p ^ key (heads of 64: p ^ key / 2), a column's eight key slots at o ^ column / 2.
    // 16 rows' pieces of one number lie in different banks then, and a piece's address is one of few bases with an exclusive or.
    auto k_place = [](int key, int piece) { return key * (HD * 2) + ((piece ^ (HD == 128 ? key & 15 : key >> 1 & 7)) << 4); };
    auto v_place = [](int col, int oct) { return L::K_BYTES + col * 128 + ((oct ^ (col >> 1 & 7)) << 4); };
    const int k_put = k_place(k_key, k_at / 8), v_put = v_place(v_col, v_oct), k_get = k_place(n16, g4), v_get = v_place(n16, g4);

    for (int tile = tile0; tile * ROWS < n; tile += tiles) {
        const int i0 = tile * ROWS, i1 = min(i0 + ROWS, n) - 1;
        const int pos_lo = p0 + i0 / G, pos_hi = p0 + i1 / G;
        KeySteps<64> ks = key_steps<64>(pos_lo, pos_hi, window, sinks);
        if (seq.over) ks.n = 0;
        const int c0 = split * chunk, c1 = split == splits - 1 ? ks.n : min(ks.n, c0 + chunk);
        const int w0 = i0 + 32 * wave, w1 = min(w0 + 31, i1);                                 // this wave's rows
        const int w_lo = p0 + min(w0, i1) / G, w_hi = w0 > i1 ? -1 : p0 + w1 / G;
        bf16x8 qf[2][QC];
        int pos[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = w0 + 16 * r + n16;
            pos[r] = i < n ? p0 + i / G : -1;
            const bf16_t* p = q + (size_t(g * G + (i < n ? i % G : 0)) * v.n_rows + seq.row0 + (i < n ? i / G : 0)) * HD + g4 * 8;
#pragma unroll
            for (int c = 0; c < QC; ++c) qf[r][c] = *(const bf16x8*)(p + 32 * c);
        }
        f32x4 acc[2][HB];
        float m[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < HB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        int e_acc = 0;

        // ---- a tile's way from memory through registers into LDS
        unsigned raw[CPT / 4];
        float sc1 = 0.f;                                       // key `lane`'s scale, of the key (wave 0) or the value (wave 1)
        bool bad = false;
        int phys = 0, off = -64, pg = 0, e_now = 0, e_most = -1000;
        auto look_up = [&](int i) {                            // tiles are looked up in their order
            off += 64;
            if (off >= v.page_tokens) { off -= v.page_tokens; ++pg; }
            if (i == c0 || i == ks.sink_steps) { pg = ks.at(i) * 64 / v.page_tokens; off = ks.at(i) * 64 - pg * v.page_tokens; }
            phys = uniform(v.table, size_t(s) * v.pages_per_seq + pg);
        };
        const unsigned k_from = k_key * HD + k_at, v_from = v_key * HD + v_col;
        auto load = [&](auto keys_) {
            bad = phys < 0 || phys >= v.n_phys;
            const unsigned char* page = v.base + size_t(bad ? 0 : phys) * v.page_bytes;
            const unsigned char* codes = page + (decltype(keys_)::value ? 0 : v.half_bytes) + (size_t(g) * v.page_tokens + off) * HD;
            if constexpr (decltype(keys_)::value) {
#pragma unroll
                for (int c = 0; c < CPT / 16; ++c) *(uint4*)&raw[4 * c] = *(const uint4*)(codes + k_from + 16 * c);
                if (wave < 2)
                    sc1 = ((const float*)(page + wave * v.half_bytes + v.scales_off))[unsigned(g * v.page_tokens + off + lane) >> (NS == 4 ? 0 : v.scale_shift)];
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const unsigned char* p = codes + v_from + (t < 4 ? t : t + 12) * HD;
                    if constexpr (VC == 8) *(uint2*)&raw[2 * t] = *(const uint2*)p;
                    else raw[t] = *(const unsigned*)p;
                }
            }
        };
        auto stage = [&](auto keys_, int c, int buf) {         // piece c of VC: eight keys' elements or a column
            unsigned char* base = lds + buf * L::TILE;
            if constexpr (decltype(keys_)::value) {
                *(bf16x8*)(base + (k_put ^ (c << 4))) = codes8(raw[2 * c], raw[2 * c + 1]);
            } else {
                auto val = [&](int t) { return code(VC == 8 ? raw[2 * t + c / 4] : raw[t], c & 3); };
                const uint4 x = {pack_code(val(0), val(1)), pack_code(val(2), val(3)), pack_code(val(4), val(5)), pack_code(val(6), val(7))};
                *(uint4*)(base + (v_put ^ (c >> 1 << 4)) + c * 128) = x;
            }
        };
        auto stage_scales = [&](int i, int slot) {             // the keys' by the first wave, the values' by the second
            if (wave == 0) {
                ((float*)(lds + L::KSC))[slot * 64 + lane] = bad ? __uint_as_float(0x7fc00000u) : sc1 * scale_log2;
            } else if (wave == 1) {
                const bool mine = visible(ks.at(i) * 64 + lane, pos_lo, pos_hi, window, sinks), fine = fabsf(sc1) <= FLT_MAX;   // mine: any row's
                const float x = mine & fine ? sc1 : 0.f;
                const unsigned long long mask = __builtin_amdgcn_ballot_w64(mine & !fine);
                const unsigned bits = __builtin_amdgcn_readfirstlane(__float_as_uint(max4(max16(fabsf(x)))));
                if (bits) {
                    const int e = int(bits >> 23) - 127;
                    e_most = max(e_most, e);
                    if (e > e_now + 3 || e < e_now - 3) e_now = max(e, e_most - 80);
                }
                ((float*)(lds + L::VSC))[slot * 64 + lane] = x * ldexpf(1.f, -e_now);
                if (lane == 0) *(int4*)(lds + L::INFO + slot * 16) = int4{e_now, 0, int(unsigned(mask)), int(unsigned(mask >> 32))};
            }
        };
        // ---- a tile's products: scores S^T = K Q^T, and O^T += V^T W^T with the weights of the tile before
        f32x4 sc[4][2];
        f16x8 wf[2][2];
        // An operand read from LDS serves two products.  AHEAD of them are on their way while others are multiplied; the fixed
        // order keeps the compiler from reading each where it is needed, where it waits for it.
        // Two chains of sums side by side, each for both blocks of rows: four products between a sum's next.
        auto key_block = [](int x) { return x / (2 * QC) * 2 + (x & 1); };
        auto key_part = [](int x) { return (x >> 1) % QC; };
        auto value_block = [](int x) { return (x >> 2) * 2 + (x & 1); };
        auto value_part = [](int x) { return (x >> 1) & 1; };
        auto key_operand = [&](int buf, int x) { return *(const bf16x8*)(lds + buf * L::TILE + (k_get ^ (key_part(x) << 6)) + key_block(x) * (16 * HD * 2)); };
        auto value_operand = [&](int buf, int x) { return *(const bf16x8*)(lds + buf * L::TILE + (v_get ^ (value_part(x) << 6)) + value_block(x) * 2048); };
        // The scores' come first: theirs are asked for before the phase begins (early).  between(x): what the vector ALUs do after
        // product x.
        constexpr int AHEAD = 4;
        bf16x8 f[AHEAD];
        auto early = [&](int buf) {
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) f[x] = key_operand(buf, x);
        };
        auto products = [&](auto fresh_, int buf, auto old_, int old_buf, auto between) {
            constexpr int K = decltype(fresh_)::value ? 4 * QC : 0, N = K + (decltype(old_)::value ? 2 * HB : 0);
            auto operand = [&](int x) { return x < K ? key_operand(buf, x) : value_operand(old_buf, x - K); };
            if constexpr (K == 0)
#pragma unroll
                for (int x = 0; x < AHEAD; ++x) f[x] = operand(x);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < N; ++x) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (x < K) {
                        f32x4& d = sc[key_block(x)][r];
                        d = mfma16(f[x % AHEAD], qf[r][key_part(x)], key_part(x) ? d : f32x4{0.f, 0.f, 0.f, 0.f});
                    } else {
                        f32x4& d = acc[r][value_block(x - K)];
                        d = mfma16h(__builtin_bit_cast(f16x8, f[x % AHEAD]), wf[r][value_part(x - K)], d);
                    }
                }
                if (x + AHEAD < N) f[x % AHEAD] = operand(x + AHEAD);
                between(x, N);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto unit_of = [&](int e_tile) {      // the outputs in the tile's units
            if (e_tile == e_acc) return;
            const float f = ldexpf(1.f, max(e_acc - e_tile, -126));
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int j = 0; j < HB; ++j) acc[r][j] *= f;
            e_acc = e_tile;
        };
        // ---- the weights of a tile from its scores
        struct Side { float4 ksc[4], vsc[4]; int4 info; };     // what LDS holds beside the operands
        auto side = [&](int slot) {
            Side d;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                d.ksc[h] = *(const float4*)(lds + L::KSC + slot * 256 + 64 * h + 16 * g4);
                d.vsc[h] = *(const float4*)(lds + L::VSC + slot * 256 + 64 * h + 16 * g4);
            }
            d.info = *(const int4*)(lds + L::INFO + slot * 16);
            return d;
        };
        auto weights = [&](auto first_, int i, const Side& d) {
            constexpr bool FIRST = decltype(first_)::value;
            const int key0 = ks.at(i) * 64;
            const bool odd = __builtin_amdgcn_readfirstlane(d.info.z | d.info.w) != 0;
            const bool edge = key0 + 63 > w_lo || w1 - w0 < 31 || (key0 <= w_hi - window && key0 + 63 >= sinks);
            auto seen = [&](int key, int r) { return visible(key, pos[r], pos[r], window, sinks); };
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    sc[h][r][0] = __builtin_fmaf(sc[h][r][0], d.ksc[h].x, -m[r]); sc[h][r][1] = __builtin_fmaf(sc[h][r][1], d.ksc[h].y, -m[r]);
                    sc[h][r][2] = __builtin_fmaf(sc[h][r][2], d.ksc[h].z, -m[r]); sc[h][r][3] = __builtin_fmaf(sc[h][r][3], d.ksc[h].w, -m[r]);
                }
            if (edge) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[h][r][e] = seen(key0 + 16 * h + 4 * g4 + e, r) ? sc[h][r][e] : -INFINITY;
            }
            if (odd) {       // values that are not finite
                const unsigned long long all = unsigned(d.info.z) | (unsigned long long)unsigned(d.info.w) << 32;
                for (int k = g4; k < 64; k += 4)
                    if (all >> k & 1)
#pragma unroll
                        for (int r = 0; r < 2; ++r) l[r] = seen(key0 + k, r) ? __uint_as_float(0x7fc00000u) : l[r];
            }
            float top[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = fmaxf(fmaxf(sc[0][r][0], sc[0][r][1]), fmaxf(sc[0][r][2], sc[0][r][3]));
#pragma unroll
                for (int h = 1; h < 4; ++h) top[r] = fmaxf(fmaxf(top[r], fmaxf(sc[h][r][0], sc[h][r][1])), fmaxf(sc[h][r][2], sc[h][r][3]));
            }
            // a row's reference moves when a weight would pass the largest, and when it sees its first keys
            auto moves = [&](int r) { return top[r] > W_TOP || (l[r] == 0.f && top[r] > -INFINITY); };
            if (FIRST || __builtin_amdgcn_ballot_w64(moves(0) || moves(1))) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float t = max4(top[r]);
                    const bool none = FIRST || sum4(l[r]) == 0.f;      // nothing summed yet, so nothing to rescale: the factor of a low t would be infinite
                    const float by = t > W_TOP || (none && t > -INFINITY) ? t - W_FIRST : 0.f, f = none ? 0.f : __builtin_amdgcn_exp2f(-by);
                    m[r] += by;
                    if constexpr (!FIRST) {
                        l[r] *= f;
#pragma unroll
                        for (int j = 0; j < HB; ++j) acc[r][j] *= f;
                    }
#pragma unroll
                    for (int h = 0; h < 4; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[h][r][e] -= by;
                }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[h][r][e] = __builtin_amdgcn_exp2f(sc[h][r][e]);
                        l[r] += sc[h][r][e];
                    }
                    sc[h][r][0] *= d.vsc[h].x; sc[h][r][1] *= d.vsc[h].y; sc[h][r][2] *= d.vsc[h].z; sc[h][r][3] *= d.vsc[h].w;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint4 x = {pack_half(sc[2 * c][r][0], sc[2 * c][r][1]), pack_half(sc[2 * c][r][2], sc[2 * c][r][3]),
                                     pack_half(sc[2 * c + 1][r][0], sc[2 * c + 1][r][1]), pack_half(sc[2 * c + 1][r][2], sc[2 * c + 1][r][3])};
                    wf[r][c] = __builtin_bit_cast(f16x8, x);
                }
            }
        };
        // Phases with a barrier between them: the first half of the waves multiplies while the second makes weights, and the other
        // way round; a SIMD has a wave of each.  In terms of the first half's tile t: phase 2t multiplies values t - 1 and keys t and, between
        // the products, converts keys t + 1; phase 2t + 1 makes the weights of tile t.  The second half is a phase behind, and
        // converts values t between its products in phase 2t + 1.  Two buffers of each and three of the scales: all are written a
        // phase or more after their last reader.
        const int nt = c1 - c0;
        auto run = [&](auto keys_) {
            constexpr bool KEYS = decltype(keys_)::value;
            constexpr int NEXT = KEYS ? 1 : 0;             // converts tile t + NEXT
            const std::true_type yes{};
            const std::false_type no{};
            look_up(c0);
            load(keys_);
            if constexpr (KEYS) {
#pragma unroll
                for (int c = 0; c < VC; ++c) stage(keys_, c, 0);
                stage_scales(c0, 0);
                if (nt > 1) { look_up(c0 + 1); load(keys_); }
                if (nt > 2) look_up(c0 + 2);
            } else {
                if (nt > 1) look_up(c0 + 1);
                phase_end();
            }
            phase_end();
            int e_next = 0, slot = 0;                      // slot: t % 3
            auto phases = [&](auto old, int t) {
                const int buf = t & 1, after = slot == 2 ? 0 : slot + 1;
                products(yes, buf, old, buf ^ 1, [&](int x, int n) {
                    const int every = n / 2 / VC, c = (x - n / 2) / every;      // from half way on: the loads are a phase old
                    if (x >= n / 2 && (x - n / 2) % every == 0 && c < VC) stage(keys_, c, KEYS ? buf ^ 1 : buf);
                });
                phase_end();
                if (KEYS && t + 1 < nt) stage_scales(c0 + t + 1, after);
                if (t + NEXT + 1 < nt) load(keys_);        // what was loaded is in LDS: the tile after it,
                if (t + NEXT + 2 < nt) look_up(c0 + t + NEXT + 2);   // and where the next one is
                const Side d = side(slot);
                __builtin_amdgcn_sched_barrier(0);
                weights(std::integral_constant<bool, !decltype(old)::value>{}, c0 + t, d);
                e_next = __builtin_amdgcn_readfirstlane(d.info.x);
                slot = after;
                if (t + 1 < nt) early(buf ^ 1);
                phase_end();
            };
            early(0);
            phases(no, 0);
            for (int t = 1; t < nt; ++t) {
                unit_of(e_next);
                phases(yes, t);
            }
            unit_of(e_next);
            products(no, 0, yes, (nt - 1) & 1, [](int, int) {});
            if (KEYS) phase_end();
            phase_end();
        };
        if (nt > 0) {
            if (keys_half) run(std::true_type{});
            else run(std::false_type{});
        }
        const float unit = ldexpf(1.f, e_acc);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = w0 + 16 * r + n16;
            float sum = sum4(l[r]);
            if (seq.over) sum = __uint_as_float(0x7fc00000u);
            if (i >= n || i > i1) continue;
            const int trow = seq.row0 + i / G, head = g * G + i % G;
            if (splits == 1) {
                const float inv = sum == 0.f ? 0.f : unit / sum;
                bf16_t* d = out + (size_t(trow) * n_q + head) * HD + 4 * g4;
#pragma unroll
                for (int j = 0; j < HB; ++j) {
                    typename Vec<bf16_t, 4>::type o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = bf16_t(acc[r][j][e] * inv);
                    *(typename Vec<bf16_t, 4>::type*)(d + 16 * j) = o;
                }
            } else {
                float* d = part + ((size_t(trow) * n_q + head) * splits + split) * (HD + 4);
                if (sum != 0.f)
#pragma unroll
                    for (int j = 0; j < HB; ++j)
                        *(float4*)(d + 16 * j + 4 * g4) = make_float4(acc[r][j][0] * unit, acc[r][j][1] * unit, acc[r][j][2] * unit, acc[r][j][3] * unit);
                if (g4 == 0) { d[HD] = sum == 0.f ? -FLT_MAX : m[r]; d[HD + 1] = sum; }
            }
        }
    }
}

// part[row][head][split][HD + 4] (unnormalised output, reference of the exponentials, sum) -> out; rows outside the batch's
// sequences are left as they are.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
merge_q8_kernel(const float* __restrict__ part, T* __restrict__ out, Q8View v, int n_q, int splits) {
    constexpr int E = HD / 16;
    const size_t i = size_t(blockIdx.x) * 16 + (threadIdx.x >> 4);
    const int e0 = (threadIdx.x & 15) * E, row = int(i / n_q);
    if (row < v.row_begin[0] || row >= min(v.row_begin[v.n_seqs], v.n_rows)) return;
    const float* p = part + i * splits * (HD + 4);
    float m = -FLT_MAX, sum = 0.f, o[E] = {};
    int used = 0;                                // ranges up to the last that has keys
    for (int b = 0; b < splits; b += 16) {       // a lane per range
        const int s = b + (threadIdx.x & 15);
        const float2 ml = s < splits ? *(const float2*)(p + size_t(s) * (HD + 4) + HD) : make_float2(-FLT_MAX, 0.f);
        float top = ml.x;
        int last = ml.y != 0.f ? s + 1 : 0;
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            top = fmaxf(top, __shfl_xor(top, d, 16));
            last = max(last, __shfl_xor(last, d, 16));
        }
        m = fmaxf(m, top);
        used = max(used, last);
    }
#pragma unroll 4
    for (int s = 0; s < used; ++s) {
        const float* ps = p + size_t(s) * (HD + 4);
        const float2 ml = *(const float2*)(ps + HD);
        const float f = __builtin_amdgcn_exp2f(ml.x - m);
        sum += ml.y * f;
        float x[E];
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 w = *(const float4*)(ps + e0 + e);
            x[e] = w.x; x[e + 1] = w.y; x[e + 2] = w.z; x[e + 3] = w.w;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += ml.y == 0.f ? 0.f : x[e] * f;   // a range without keys has left nothing
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    typename Vec<T, E>::type ov;
#pragma unroll
    for (int e = 0; e < E; ++e) ov[e] = to_elem<T>(o[e] * inv);
    *(typename Vec<T, E>::type*)(out + i * HD + e0) = ov;
}

// A sequence's tiles beyond the launch's go round again, so a hint that is too small costs time and one that is too large none.
constexpr int MOST_GROUPS = 1 << 18;

template <typename T, int HD>
hipError_t append_q8(const float* qkv, T* q, T* values, const Q8View& v, const cake_rope& rope, int n_q, int max_rows, hipStream_t st) {
    const int most = std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv)), heads = v.scale_shift ? n_q : n_q + 2 * v.n_kv;
    const int row_tiles = std::min((max_rows + 7) / 8, most), block_tiles = v.scale_shift ? std::min((max_rows + 63) / 64 + 1, most) : 0;
    // few rows: their heads on several workgroups, down to one row of a head per sixteen lanes
    const int chunks = std::max(1, std::min((heads * std::min(max_rows, 8) + 15) / 16, 1024 / (v.n_seqs * row_tiles)));
    const int row_groups = v.n_seqs * row_tiles * chunks, block_groups = v.n_seqs * block_tiles * v.n_kv;
    auto go = [&](auto mode) {
        hipLaunchKernelGGL((append_q8_kernel<T, HD, decltype(mode)::value>), dim3(unsigned(row_groups + block_groups)), dim3(256), 0, st, qkv, q, values, v, rope,
                           n_q, row_tiles, chunks, block_groups, block_tiles);
        return hipGetLastError();
    };
    if (rope.layout == CAKE_ROPE_PAIRS) return go(std::integral_constant<int, ROPE_ADJACENT>{});
    if (rope.rotary_dim == HD) return go(std::integral_constant<int, ROPE_HALVES>{});
    return go(std::integral_constant<int, ROPE_HALVES_PART>{});
}

// How a launch divides the keys: `chunk` steps of `width` keys to a workgroup, at most `splits` ranges.  About `want` workgroups
// of `least` steps or more.  Tiles of 16 and 32 rows: 2048 of 4 to 48 steps (64 ragged sequences up to 8191 keys, with the merge:
// 4 steps 158 us, 12 144, 24 133, 32 138, 48 133, 64 149, 129 155; one of 701: 4 steps 10.1, 8 11.2, 24 13.1 without a merge).
// Tiles of 128 rows: 512, two a compute unit (16 ragged sequences, 128 rows: 256 116 us, 512 81, 1024 87); of 256: 256 (one of
// 16000 keys: 256 48 us, 512 65).
// In tiles of 128 and 256 rows the workgroups are those that can have rows: a ragged batch has no more tiles than its rows fill and one for
// each sequence's last.  Measured (us, as if every sequence had max_rows rows, and so; 8 KV heads of 128, one chunk beside single
// tokens): 256 rows, three tokens, all at 16000 keys 419, 221; 256 rows at 8000, 15 tokens at 500 to 8191 689, 421; 1024 rows, three
// tokens at 16000 819, 726; 1024 rows at 8000, three tokens at 500 to 8191 367, 380; 63 tokens 2144, 2144.  Tiles of 16 and 32 rows are many small
// workgroups, and those without rows count in what a launch takes: 24 rows at 8000, three tokens 32, 41, so there it is all of them.
struct KeyRanges { int tiles, chunk, splits; int64_t steps, groups; };
KeyRanges key_ranges(const Q8View& v, int n_q, int rows_per_tile, int width, int max_rows, int max_len, int window, int sinks, int least, int most, int64_t want,
                     const AttnWs& ws) {
    KeyRanges k;
    const int G = n_q / v.n_kv;
    k.tiles = int(std::min<int64_t>((int64_t(max_rows) * G + rows_per_tile - 1) / rows_per_tile, std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv))));
    const int64_t seen = std::min<int64_t>(max_len, int64_t(window) + sinks + rows_per_tile / G + 2 * width);
    const int64_t steps = k.steps = seen / width + 1;
    k.groups = int64_t(v.n_seqs) * v.n_kv * k.tiles;
    const int64_t busy = rows_per_tile < 128 ? k.groups : v.n_kv * std::min<int64_t>(int64_t(v.n_seqs) * k.tiles, int64_t(v.n_rows) * G / rows_per_tile + v.n_seqs);
    int64_t chunk = std::min<int64_t>(std::max<int64_t>(least, (steps * busy + want - 1) / want), most);
    chunk = std::max(chunk, steps * k.groups / 16384);        // ranges past a sequence's end cost a little too
    int64_t splits = std::max<int64_t>(1, (steps + chunk - 1) / chunk);
    splits = std::min<int64_t>(splits, int64_t(ws.bytes / (size_t(v.n_rows) * n_q * (v.head_dim + 4) * 4)));
    if (splits < 1) splits = 1;
    k.chunk = int((steps + splits - 1) / splits);
    k.splits = int(splits);
    return k;
}

template <typename T>
hipError_t merge_q8(const Q8View& v, int n_q, const KeyRanges& k, const AttnWs& ws, T* out, hipStream_t st) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || k.splits == 1) return e;
    const dim3 grid(unsigned((size_t(v.n_rows) * n_q + 15) / 16));
    if (v.head_dim == 128) hipLaunchKernelGGL((merge_q8_kernel<T, 128>), grid, dim3(256), 0, st, ws.part, out, v, n_q, k.splits);
    else hipLaunchKernelGGL((merge_q8_kernel<T, 64>), grid, dim3(256), 0, st, ws.part, out, v, n_q, k.splits);
    return hipGetLastError();
}

template <typename T, int HD, int NB, int NS>
hipError_t attention_q8(const T* q, T* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks, float scale, const AttnWs& ws, hipStream_t st) {
    const KeyRanges k = key_ranges(v, n_q, 16 * NB, 32, max_rows, max_len, window, sinks, 4, 48, 2048, ws);
    // Undivided on eight waves, without a merge, where sequences are not too long for it: one such workgroup fills a compute unit, so the
    // steps that may be walked by one grow with the share of the 256 units that the last of up to two rounds fills.  Measured (us,
    // against four waves, divided, with the merge; a token each, 8 KV heads of 128, then of 64; sequences x keys): 1 x 300 7.5, 9.0;
    // 1 x 701 11.1, 9.6; 8 x 1500 18.9, 14.4; 16 x 2000 23.1, 24.7 and 16.8, 17.1; 16 x 5000 54.9, 46.9 and 34.5, 26.5;
    // 24 x 4100 47.2, 53.8 and 32.9, 32.7; 32 x 2000 31.3, 38.0 and 17.4, 21.6; 32 x 4100 56.5, 66.5 and 34.3, 39.5;
    // 33 x 300 14.7, 14.7 and 8.1, 10.7; 33 x 2000 49.3, 41.1 and 24.3, 23.7; 33 x 4100 89.8, 69.3 and 45.6, 41.4; 36 x 1500 39.6, 35.0 and
    // 19.9, 20.8; 48 x 1000 31.0, 33.5 and 16.1, 21.2; 48 x 3000 74.5, 69.2 and 38.5, 41.5; 64 x 4100 107.6, 116.3 and 59.0, 66.0.
    // Longer ones of equal length gain too (32 x 8191 105, 114), ragged ones lose what the longest takes alone: 32 of 500 to 4100 44.0,
    // 44.1, to 8191 84.5, 86.0 and 57.9, 51.6, to 30000 284, 238 and 194, 134; hence no more than 12 + 256 * 256 / 550 steps.
    // Two workgroups of tiles of 16 rows, heads of 64 and two-byte elements fit a unit: 50 steps in a second round that is hardly filled.
    constexpr bool PAIRS = HD == 64 && NB == 1 && Terms<T>::Q == 1;
    const int64_t last = k.groups % 256 ? k.groups % 256 : 256, by_fill = 12 + last * last / 550;
    const int64_t most_steps = k.groups > 512 ? 0 : PAIRS && k.groups > 256 ? std::max<int64_t>(50, by_fill) : by_fill;
    if (k.steps <= most_steps) {
        hipLaunchKernelGGL((attention_q8_kernel<T, HD, NB, NS, 8>), dim3(unsigned(k.groups)), dim3(512), 0, st, q, out, ws.part, v, n_q, window, sinks, scale,
                           int(k.steps), 1, k.tiles);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((attention_q8_kernel<T, HD, NB, NS, 4>), dim3(unsigned(k.groups * k.splits)), dim3(256), 0, st, q, out, ws.part, v, n_q, window, sinks,
                       scale, k.chunk, k.splits, k.tiles);
    return merge_q8(v, n_q, k, ws, out, st);
}

template <int HD, int NWV, int NS>
hipError_t attention_q8_rows(const bf16_t* q, bf16_t* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks, float scale, const AttnWs& ws,
                             hipStream_t st) {
    const KeyRanges k = key_ranges(v, n_q, 32 * NWV, 64, max_rows, max_len, window, sinks, 4, 1 << 20, NWV == 8 ? 256 : 512, ws);
    constexpr int LDS = RowsLds<HD>::BYTES;
    static std::atomic<uint64_t> set{0};                       // a bit per device
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess && !(set.load(std::memory_order_relaxed) >> (device & 63) & 1)) {
        e = hipFuncSetAttribute((const void*)attention_q8_rows_kernel<HD, NWV, NS>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e == hipSuccess) set.fetch_or(uint64_t(1) << (device & 63), std::memory_order_relaxed);
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attention_q8_rows_kernel<HD, NWV, NS>), dim3(unsigned(k.groups * k.splits)), dim3(64 * NWV), LDS, st, q, out, ws.part, v, n_q, window,
                       sinks, scale, k.chunk, k.splits, k.tiles);
    return merge_q8(v, n_q, k, ws, out, st);
}
}  // namespace

hipError_t launch_append_q8(int dtype, const float* qkv, void* q, void* values, const Q8View& v, const cake_rope& rope, int n_q, int max_rows, hipStream_t st) {
    if (dtype == CAKE_F32)
        return v.head_dim == 128 ? append_q8<float, 128>(qkv, (float*)q, (float*)values, v, rope, n_q, max_rows, st)
                                 : append_q8<float, 64>(qkv, (float*)q, (float*)values, v, rope, n_q, max_rows, st);
    return v.head_dim == 128 ? append_q8<bf16_t, 128>(qkv, (bf16_t*)q, (bf16_t*)values, v, rope, n_q, max_rows, st)
                             : append_q8<bf16_t, 64>(qkv, (bf16_t*)q, (bf16_t*)values, v, rope, n_q, max_rows, st);
}

hipError_t launch_attention_q8(int dtype, const void* q, void* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks,
                               const AttnWs& ws, hipStream_t st) {
    const int64_t rows = int64_t(max_rows) * (n_q / v.n_kv);
    window = window == 0 ? Q8_MOST_TOKENS : std::min(window, Q8_MOST_TOKENS);   // none: longer than any sequence, and position - window stays a number
    const float scale = 1.44269504088896340736f / std::sqrt(float(v.head_dim));
    auto go = [&](auto hd, auto ns) {
        constexpr int HD = decltype(hd)::value, NS = decltype(ns)::value;
        if (dtype == CAKE_F32) return attention_q8<float, HD, 1, NS>((const float*)q, (float*)out, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        const bf16_t* qb = (const bf16_t*)q;
        bf16_t* ob = (bf16_t*)out;
        // Tiles of 32 rows where one holds them all: 33 sequences up to 4099, 20 rows, heads of 64: 45 us, 50 with two tiles of 16.
        if (rows > 16 && rows <= 32) return attention_q8<bf16_t, HD, 2, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        // Heads of 128: what a tile costs, in halves of a tile of 16 rows.  Measured (us; tiles of 16, of 128, of 256 rows), 32 / 8 heads:
        // 16 sequences of 8191 keys: 36 rows 82, 144, -; 96 rows 159, 145, 251; 192 rows 253, 264, 251; 256 rows 326, 266, 251;
        // 16 ragged ones up to 4099: 36 rows 40, 78, -; 128 rows 73, 81, 116; 132 rows 73, 133, 128; 256 rows 101, 140, 128;
        // 1 of 16000: 36 rows 46, 42, -; 128 rows 53, 44, -; 256 rows 79, 52, 48; 4 of 4096, 512 rows: 97, 82, 75.
        if constexpr (HD == 128) {
            const int64_t few = 2 * ((rows + 15) / 16), four = 13 * ((rows + 127) / 128), eight = 24 * ((rows + 255) / 256);
            if (four < few && four < eight) return attention_q8_rows<HD, 4, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
            if (eight <= few) return attention_q8_rows<HD, 8, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        // Heads of 64, half the bytes and products at the same other work: 1 of 16000: 192 rows 42, 45, 48; 512 rows 85, 66, 73;
        // 1024 rows 159, 109, 123; 4 of 4096: 512 rows 61, 74, 83; 1024 rows 111, 133, 133; 16 of 8191: 256 rows 194, 242, 327.
        } else if (rows >= 512) {
            return attention_q8_rows<HD, 4, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        }
        return attention_q8<bf16_t, HD, 1, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
    };
    const std::integral_constant<int, 128> hd128{};
    const std::integral_constant<int, 64> hd64{};
    const std::integral_constant<int, 4> each{};     // a scale per token: four neighbours' at once
    const std::integral_constant<int, 1> shared{};   // four tokens or more share one
    if (v.scale_shift == 0) return v.head_dim == 128 ? go(hd128, each) : go(hd64, each);
    return v.head_dim == 128 ? go(hd128, shared) : go(hd64, shared);
}

}  // namespace cake
