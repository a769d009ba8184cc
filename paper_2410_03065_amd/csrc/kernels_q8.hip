// A ragged batch over an 8-bit paged cache (layout: cake.h, cake_q8_batch): appending rotated keys and values, and
// attention that reads the codes.
//
// Key j of a KV head stands for the vector c_j * s_j: int8 codes c_j and the float32 scale s_j of the block of tokens that
// it lies in.  A score is therefore (q . c_j) * s_j and an output sum_j (p_j s'_j) c'_j: the products run on the codes as they
// are, exact in bfloat16 (eight bits), and a scale is one factor per score.  No dequantised copy of the cache exists anywhere.
#include <algorithm>
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
__device__ __forceinline__ float sum4(float y) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A sequence of the batch.  What the device arrays say is not trusted: rows stay inside [0, n_rows), and a length that the
// block table cannot hold (over) is never followed.
struct Seq { int row0, rows, len; bool over; };
__device__ __forceinline__ Seq sequence(const Q8View& v, int s) {
    Seq q;
    q.row0 = min(max(v.row_begin[s], 0), v.n_rows);
    q.rows = min(max(v.row_begin[s + 1], q.row0), v.n_rows) - q.row0;
    q.len = min(max(v.seq_len[s], 0), Q8_MOST_TOKENS);
    q.over = q.len > v.pages_per_seq * v.page_tokens;
    return q;
}

template <typename T> __device__ __forceinline__ T to_elem(float x);
template <> __device__ __forceinline__ float to_elem<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t to_elem<bf16_t>(float x) { return bf16_t(x); }

template <typename T, int N> struct Vec { typedef T type __attribute__((__vector_size__(N * sizeof(T)))); };

// ===================================================================================== append
// Workgroup: `tile` positions of a sequence (a multiple of the block of tokens that shares a scale, aligned to it, so no two
// workgroups write one block) and one KV head with the query heads of its group.  Sixteen lanes hold a head's row.
// Bound by the bytes: 4 read per element and 1 or 2 written; the rotation runs in 64 bits (full rate on this chip), because
// at position 60000 a float32 angle is off by 4e-3 and because the codes that follow are whole numbers: with the rotated
// value correctly rounded to float32 they do not depend on how cosine and sine were come by.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
append_q8_kernel(const float* __restrict__ qkv, T* __restrict__ q, T* __restrict__ values, Q8View v, cake_rope rope, int n_q, int tile, int tiles) {
    constexpr int E = HD / 16;                      // elements per lane
    typedef typename Vec<T, E>::type TV;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    double2* cs = (double2*)lds;                    // [tile][HD / 2]
    unsigned* amax = (unsigned*)(lds + size_t(tile) * (HD / 2) * sizeof(double2));   // [K|V][tile]: a block's largest magnitude, then its scale
    float* ratio = (float*)(amax + 2 * tile);       // [K|V]: what the codes of the first block's older tokens are multiplied by
    const int g = blockIdx.x % v.n_kv, t_first = blockIdx.x / v.n_kv % tiles, s = blockIdx.x / v.n_kv / tiles;
    const int G = n_q / v.n_kv, heads = G + 2, all_heads = n_q + 2 * v.n_kv;
    const int tid = threadIdx.x, group = tid >> 4, e0 = (tid & 15) * E;
    const Seq seq = sequence(v, s);
    const int p0 = seq.len - seq.rows, half = rope.rotary_dim / 2, block = 1 << v.scale_shift;
    const int cap = v.pages_per_seq * v.page_tokens;
    const int p_new = max(p0, 0), base0 = p_new / tile * tile;   // rows in excess of the sequence's tokens stand for no token
    const bool pairs = rope.layout == CAKE_ROPE_PAIRS;

    for (int t = t_first; base0 + t * tile < seq.len; t += tiles) {
        const int base = base0 + t * tile;
        const int lo = max(base, p_new), n = min(base + tile, seq.len) - lo;   // this tile's new positions
        if (n <= 0) return;
        if (t != t_first) __syncthreads();
        for (int i = tid; i < n * half; i += 256) {
            double sn, cn;
            sincos(double(lo + i / half) * rope.freq[i % half], &sn, &cn);
            cs[(i / half) * (HD / 2) + i % half] = double2{cn * rope.magnitude, sn * rope.magnitude};
        }
        if (block > 1)
            for (int i = tid; i < 2 * tile; i += 256) amax[i] = 0;
        __syncthreads();
        // One head's row: rotated (queries and keys) in 64 bits, rounded to float32.
        auto row_of = [&](int i, int h, float (&x)[E]) {
            const int row = seq.row0 + (lo + i - p0);
            const float* p = qkv + (size_t(row) * all_heads + (h < G ? g * G + h : h == G ? n_q + g : n_q + v.n_kv + g)) * HD;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const float4 w = *(const float4*)(p + e0 + e);
                x[e] = w.x; x[e + 1] = w.y; x[e + 2] = w.z; x[e + 3] = w.w;
            }
            if (h > G) return;
            const double2* c = cs + i * (HD / 2);
            if (pairs) {
#pragma unroll
                for (int e = 0; e < E; e += 2)
                    if (e0 + e < rope.rotary_dim) {
                        const double2 z = c[(e0 + e) / 2];
                        const double a = x[e], b = x[e + 1];
                        x[e] = float(a * z.x - b * z.y);
                        x[e + 1] = float(a * z.y + b * z.x);
                    }
            } else if (e0 < rope.rotary_dim) {
                float y[E] = {};
                if (half % E == 0) {            // the partners lie side by side too
                    const float* o = p + (e0 < half ? e0 + half : e0 - half);
#pragma unroll
                    for (int e = 0; e < E; e += 4) {
                        const float4 w = *(const float4*)(o + e);
                        y[e] = w.x; y[e + 1] = w.y; y[e + 2] = w.z; y[e + 3] = w.w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e0 + e < rope.rotary_dim) y[e] = p[e0 + e < half ? e0 + e + half : e0 + e - half];
                }
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e0 + e < rope.rotary_dim) {
                        const bool first = e0 + e < half;
                        const double2 z = c[first ? e0 + e : e0 + e - half];
                        x[e] = float(first ? double(x[e]) * z.x - double(y[e]) * z.y : double(x[e]) * z.x + double(y[e]) * z.y);
                    }
            }
        };
        // the row's largest magnitude, as bits: they order like the numbers, and infinities and NaN come out on top
        auto largest = [&](const float (&x)[E]) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
            for (int o = 8; o; o >>= 1) m = max(m, unsigned(__shfl_xor(int(m), o, 16)));
            return m;
        };
        auto scale_of = [](unsigned m) { return m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(m) / 127.0f; };
        auto page_of = [&](int pos) -> unsigned char* {   // null where nothing can be written
            if (pos >= cap) return nullptr;
            const int phys = v.table[size_t(s) * v.pages_per_seq + pos / v.page_tokens];
            return phys < 0 || phys >= v.n_phys ? nullptr : v.base + size_t(phys) * v.page_bytes;
        };
        auto put = [&](int i, int which, const float (&x)[E], float scale, unsigned char* page) {
            const int pos = lo + i, off = pos % v.page_tokens;
            float c[E];
            unsigned w[E / 4] = {};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                c[e] = scale > 0.f ? fminf(fmaxf(rintf(x[e] / scale), -127.f), 127.f) : 0.f;
                w[e / 4] |= (unsigned(int(c[e])) & 255u) << (8 * (e & 3));
            }
            if (page) {
                unsigned char* half_page = page + which * v.half_bytes;
                unsigned* d = (unsigned*)(half_page + (size_t(g) * v.page_tokens + off) * HD + e0);
#pragma unroll
                for (int e = 0; e < E / 4; ++e) d[e] = w[e];
                if (block == 1 && e0 == 0) ((float*)(half_page + v.scales_off))[size_t(g) * v.page_tokens + off] = scale;
            }
            if (values) {
                TV o;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = to_elem<T>(page ? c[e] * scale : __uint_as_float(0x7fc00000u));
                *(TV*)(values + (size_t(seq.row0 + pos - p0) * 2 * v.n_kv + which * v.n_kv + g) * HD + e0) = o;
            }
        };
        if (block > 1) {      // a block's scale first: its largest magnitude, over its older tokens' scale too
            for (int i = group; i < 2 * n; i += 16) {
                float x[E];
                const int which = i & 1, tok = i >> 1, pos = lo + tok;
                row_of(tok, G + which, x);
                const unsigned a = largest(x);
                if (e0 == 0) atomicMax(&amax[which * tile + ((pos - base) >> v.scale_shift)], a);
            }
            __syncthreads();
            const int blocks = tile >> v.scale_shift;
            for (int i = tid; i < 2 * blocks; i += 256) {
                const int which = i & 1, b = i >> 1, start = base + (b << v.scale_shift);
                float scale = scale_of(amax[which * tile + b]);
                unsigned char* page = start < lo + n && start + block > lo ? page_of(start) : nullptr;
                if (page) {
                    float* where = (float*)(page + which * v.half_bytes + v.scales_off) +
                                   ((size_t(g) * v.page_tokens + start % v.page_tokens) >> v.scale_shift);
                    if (start < lo) {
                        const float old = *where;
                        if (!(old <= scale)) scale = old;                 // also where either is NaN
                        if (amax[which * tile + b] >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);
                        ratio[which] = scale > 0.f ? old / scale : 1.f;
                    }
                    *where = scale;
                }
                amax[which * tile + b] = __float_as_uint(scale);
            }
            __syncthreads();
            const int start = lo / block * block;            // the older tokens of the first block
            if (start < lo) {
                unsigned char* page = page_of(start);
                const int words = (lo - start) * (HD / 4);
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
            }
        }
        for (int i = group; i < n * heads; i += 16) {
            const int tok = i / heads, h = i - tok * heads, pos = lo + tok;
            float x[E];
            row_of(tok, h, x);
            if (h < G) {
                TV o;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = to_elem<T>(x[e]);
                *(TV*)(q + (size_t(g * G + h) * v.n_rows + seq.row0 + pos - p0) * HD + e0) = o;
            } else {
                const int which = h - G;
                float scale;
                if (block > 1) scale = __uint_as_float(amax[which * tile + ((pos - base) >> v.scale_shift)]);
                else scale = scale_of(largest(x));
                put(tok, which, x, scale, page_of(pos));
            }
        }
    }
}

// ===================================================================================== attention
// The keys that some row of a tile of rows sees, in steps of 32: the steps of the first tokens that stay visible, then from
// the window's (step number i stands for step at(i)).
struct KeySteps {
    int sink_steps, first, n;
    __device__ __forceinline__ int at(int i) const { return i < sink_steps ? i : first + i - sink_steps; }
};
__device__ __forceinline__ KeySteps key_steps(int pos_lo, int pos_hi, int window, int sinks) {
    KeySteps k = {0, 0, 0};
    if (pos_hi < 0) return k;
    if (window > 0 && pos_lo - window + 1 > 0) {
        k.first = (pos_lo - window + 1) / 32;
        k.sink_steps = (min(sinks, pos_lo - window + 1) + 31) / 32;
        if (k.sink_steps >= k.first) k.first = k.sink_steps = 0;
    }
    k.n = k.sink_steps + pos_hi / 32 + 1 - k.first;
    return k;
}

// Few rows.  A tile is NB x 16 rows (token, query head of the group) of one sequence and KV head; a workgroup takes a range of
// its key steps, its four waves every fourth step each, straight from memory into registers.  Scores are formed transposed,
// S^T[key][row] = K Q^T, so that a lane holds four keys of one row per block of 16 and the weights are the second product's
// operand as they are: O^T[hd][row] += V^T W^T, where the slots of a product are dealt to keys as the scores lie (slot
// 8g + t: key 4g + t, from t = 4 key 16 + 4g + t - 4).  A lane reads 8 (4) neighbouring elements of eight keys' values and
// its conversions pick the bytes, so nothing is transposed.  Bound by the cache's bytes; per byte 1.5 vector instructions.
// Weights go to the product as two bfloat16 values each (16 bits; float32 models: three, all 24, as the queries): at this
// size the matrix cores are idle, and a single bfloat16 would double the output's rounding error.
template <typename T> struct Terms { static constexpr int Q = 1, W = 2; };
template <> struct Terms<float> { static constexpr int Q = 3, W = 3; };

template <typename T, int HD, int NB>
__global__ void __launch_bounds__(256)
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
        KeySteps ks = key_steps(pos_lo, pos_hi, window, sinks);
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
        struct Step { uint4 k[2][KB / 16]; uint2 vv[8]; float ksc[2][4], vsc[2][4]; };
        auto load = [&](Step& st, int i) {
            const int key0 = ks.at(i) * 32, pg = key0 / v.page_tokens, off = key0 - pg * v.page_tokens;
            const int phys = v.table[size_t(s) * v.pages_per_seq + pg];
            const bool bad = phys < 0 || phys >= v.n_phys;
            const unsigned char* page = v.base + size_t(bad ? 0 : phys) * v.page_bytes;
            const unsigned char* kc = page + (size_t(g) * v.page_tokens + off) * HD;
            const unsigned char* vc = kc + v.half_bytes;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < KB / 16; ++c) st.k[h][c] = *(const uint4*)(kc + (16 * h + n16) * HD + g4 * KB + 16 * c);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const unsigned char* p = vc + ((t < 4 ? 0 : 12) + 4 * g4 + t) * HD + n16 * CW;
                if constexpr (CW == 8) st.vv[t] = *(const uint2*)p;
                else st.vv[t].x = *(const unsigned*)p;
            }
            const float* kst = (const float*)(page + v.scales_off);
            const float* vst = (const float*)(page + v.half_bytes + v.scales_off);
            const int at = g * v.page_tokens + off + 4 * g4;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (v.scale_shift == 0) {
                    *(float4*)st.ksc[h] = *(const float4*)(kst + at + 16 * h);
                    *(float4*)st.vsc[h] = *(const float4*)(vst + at + 16 * h);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        st.ksc[h][e] = kst[(at + 16 * h + e) >> v.scale_shift];
                        st.vsc[h][e] = vst[(at + 16 * h + e) >> v.scale_shift];
                    }
                }
                if (bad)     // keys of a page outside the pool: whoever sees them gets NaN
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.ksc[h][e] = __uint_as_float(0x7fc00000u);
            }
        };
        auto step = [&](const Step& st, int i) {
            const int key0 = ks.at(i) * 32;
            const bool edge = key0 + 31 > pos_lo || i1 - i0 + 1 < 16 * NB || (window > 0 && key0 <= pos_hi - window && key0 + 31 >= sinks);
            bf16x8 kf[2][QC];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    const uint4 w = st.k[h][c / 2];
                    kf[h][c] = c & 1 ? codes8(w.z, w.w) : codes8(w.x, w.y);
                }
            bf16x8 wf[NB][TW];
#pragma unroll
            for (int r = 0; r < NB; ++r) {
                f32x4 sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = TQ - 1; t >= 0; --t)
#pragma unroll
                        for (int c = 0; c < QC; ++c) sc[h] = mfma16(kf[h][c], qf[r][t][c], sc[h]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[h][e] *= st.ksc[h][e] * scale_log2;
                }
                if (edge) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + 16 * h + 4 * g4 + e;
                            const bool seen = key <= pos[r] && (window <= 0 || key > pos[r] - window || key < sinks);
                            sc[h][e] = seen ? sc[h][e] : -INFINITY;
                        }
                }
                float top = m[r];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[h][e]);
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
                        const float p = __builtin_amdgcn_exp2f(sc[h][e] - top);
                        l[r] += p;
                        // a hidden key's scale may be anything: memory behind the last token
                        float w = edge && sc[h][e] == -INFINITY ? 0.f : p * st.vsc[h][e];
#pragma unroll
                        for (int t = 0; t < TW; ++t) { wf[r][t][4 * h + e] = bf16_t(w); w -= float(wf[r][t][4 * h + e]); }
                    }
            }
#pragma unroll
            for (int j = 0; j < CW; ++j) {
                uint4 a;
                auto col = [&](int t) { return code(j < 4 ? st.vv[t].x : st.vv[t].y, j & 3); };
                a.x = pack_hi(col(0), col(1)); a.y = pack_hi(col(2), col(3)); a.z = pack_hi(col(4), col(5)); a.w = pack_hi(col(6), col(7));
                const bf16x8 vf = __builtin_bit_cast(bf16x8, a);
#pragma unroll
                for (int r = 0; r < NB; ++r)
#pragma unroll
                    for (int t = TW - 1; t >= 0; --t) acc[r][j] = mfma16(vf, wf[r][t], acc[r][j]);
            }
        };
        Step a, c;
        int i = c0 + wave;
        if (i < c1) load(a, i);
        for (; i < c1; i += 8) {
            if (i + 4 < c1) load(c, i + 4);
            step(a, i);
            if (i + 4 >= c1) break;
            if (i + 8 < c1) load(a, i + 8);
            step(c, i + 4);
        }
        // the four waves' parts, added up in their order
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            if (r) __syncthreads();
            const float lt = sum4(l[r]);
            if (g4 == 0) { s_ml[wave][n16][0] = m[r]; s_ml[wave][n16][1] = lt; }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < CW; j += 4)
                    *(float4*)&s_acc[wave][n16][(4 * g4 + e) * CW + j] = make_float4(acc[r][j][e], acc[r][j + 1][e], acc[r][j + 2][e], acc[r][j + 3][e]);
            __syncthreads();
            const int row = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * CW, idx = i0 + 16 * r + row;
            if (idx < n) {
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
    float m = -FLT_MAX;
    for (int s = 0; s < splits; ++s) m = fmaxf(m, p[s * (HD + 4) + HD]);
    float sum = 0.f, o[E] = {};
    for (int s = 0; s < splits; ++s) {
        const float l = p[s * (HD + 4) + HD + 1];
        if (l == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(p[s * (HD + 4) + HD] - m);
        sum += l * f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += p[s * (HD + 4) + e0 + e] * f;
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
    const int tile = std::max(16, 1 << v.scale_shift), tiles = std::min((max_rows + tile - 1) / tile + 1, std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv)));
    const size_t lds = size_t(tile) * (HD / 2) * sizeof(double2) + (2 * tile + 2) * 4;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)append_q8_kernel<T, HD>, hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((append_q8_kernel<T, HD>), dim3(unsigned(size_t(v.n_seqs) * tiles * v.n_kv)), dim3(256), lds, st, qkv, q, values, v, rope, n_q, tile, tiles);
    return hipGetLastError();
}

template <typename T, int HD, int NB>
hipError_t attention_q8(const T* q, T* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks, const AttnWs& ws, hipStream_t st) {
    const int G = n_q / v.n_kv, tiles = int(std::min<int64_t>((int64_t(max_rows) * G + 16 * NB - 1) / (16 * NB), std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv))));
    const int64_t seen = window > 0 ? std::min<int64_t>(max_len, int64_t(window) + sinks + 16 * NB + 64) : max_len;
    const int64_t steps = seen / 32 + 1, groups = int64_t(v.n_seqs) * v.n_kv * tiles;
    // key ranges: enough workgroups for the chip, none shorter than one step per wave
    int64_t chunk = std::max<int64_t>(4, (steps * groups + 2047) / 2048);
    int64_t splits = std::max<int64_t>(1, (steps + chunk - 1) / chunk);
    const size_t row = size_t(v.n_rows) * n_q * (HD + 4) * 4;
    splits = std::min<int64_t>(splits, ws.part ? int64_t(ws.bytes / row) : 1);
    if (splits < 1) splits = 1;
    chunk = (steps + splits - 1) / splits;
    const float scale = 1.44269504088896340736f / std::sqrt(float(HD));
    hipLaunchKernelGGL((attention_q8_kernel<T, HD, NB>), dim3(unsigned(groups * splits)), dim3(256), 0, st, q, out, ws.part, v, n_q, window, sinks,
                       scale, int(chunk), int(splits), tiles);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    hipLaunchKernelGGL((merge_q8_kernel<T, HD>), dim3(unsigned((size_t(v.n_rows) * n_q + 15) / 16)), dim3(256), 0, st, ws.part, out, v, n_q, int(splits));
    return hipGetLastError();
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
    const bool one = int64_t(max_rows) * (n_q / v.n_kv) <= 16;
    auto go = [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        if (dtype == CAKE_F32) return attention_q8<float, HD, 1>((const float*)q, (float*)out, v, n_q, max_rows, max_len, window, sinks, ws, st);
        return one ? attention_q8<bf16_t, HD, 1>((const bf16_t*)q, (bf16_t*)out, v, n_q, max_rows, max_len, window, sinks, ws, st)
                   : attention_q8<bf16_t, HD, 2>((const bf16_t*)q, (bf16_t*)out, v, n_q, max_rows, max_len, window, sinks, ws, st);
    };
    return v.head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace cake
