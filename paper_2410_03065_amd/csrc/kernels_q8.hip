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
// The keys that some row of a tile of rows sees, in steps of W: the steps of the first tokens that stay visible, then from
// the window's (step number i stands for step at(i)).
template <int W> struct KeySteps {
    int sink_steps, first, n;
    __device__ __forceinline__ int at(int i) const { return i < sink_steps ? i : first + i - sink_steps; }
};
template <int W> __device__ __forceinline__ KeySteps<W> key_steps(int pos_lo, int pos_hi, int window, int sinks) {
    KeySteps<W> k = {0, 0, 0};
    if (pos_hi < 0) return k;
    if (window > 0 && pos_lo - window + 1 > 0) {
        k.first = (pos_lo - window + 1) / W;
        k.sink_steps = (min(sinks, pos_lo - window + 1) + W - 1) / W;
        if (k.sink_steps >= k.first) k.first = k.sink_steps = 0;
    }
    k.n = k.sink_steps + pos_hi / W + 1 - k.first;
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

template <typename T, int HD, int NB, int NS>
__global__ void __launch_bounds__(256, NB == 2 || Terms<T>::Q == 3 ? 2 : HD == 128 ? 3 : 4)
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
            phys = v.table[size_t(s) * v.pages_per_seq + pg];
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
        for (; i < c1; i += 4) {
            const int key0 = ks.at(i) * 32;
            const bool more = i + 4 < c1, was_bad = bad;
            if (more) look_up(i + 4);
            const bool edge = key0 + 31 > pos_lo || i1 - i0 + 1 < 16 * NB || (window > 0 && key0 <= pos_hi - window && key0 + 31 >= sinks);
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
                            const int key = key0 + 16 * h + 4 * g4 + e;
                            const bool seen = key <= pos[r] && (window <= 0 || key > pos[r] - window || key < sinks);
                            sc[r][h][e] = seen ? sc[r][h][e] : -INFINITY;
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

// Many rows.  A workgroup takes 32 rows (token, query head of the group) per wave and tiles of 64 keys, which it converts once
// for all of them on the way into LDS, two tiles there in turn: keys as bfloat16 codes [key][hd], values transposed
// [hd][key slot] in half precision, code * scale / 2^E.  E is the exponent of the tile's largest scale (kept while it moves by
// less than 8 times; the outputs are in units of 2^E and move with it), so eleven bits of every value survive whatever the
// scales' range; scaling the values here saves a multiplication per score.  A value scale that is not finite leaves zeros and
// a bit in the tile's mask: rows that see its key get a NaN sum, the others nothing.
// Weights are exp2(score - m) in half precision up to 2^15: m follows a row's maximum only when it would pass that, so the
// output registers are hardly ever rescaled and rows exchange nothing between lanes on the way.
// Scores transposed, key slots and the operands' order as above.  Rows of 16 bytes in LDS are swizzled so that neither the
// 16 rows that a product reads nor those that a conversion writes meet in a bank.
// Bound by the vector instructions beside the products (8 a score, 2 a code over the workgroup's rows).
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
__device__ __forceinline__ f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ unsigned pack_half(float a, float b) { return __builtin_bit_cast(unsigned, f16x2{_Float16(a), _Float16(b)}); }

constexpr float W_TOP = 15.f, W_FIRST = 8.f;      // largest exponent of a weight; where a row's maximum is put

template <int HD> struct RowsLds {
    static constexpr int K_BYTES = 64 * HD * 2, TILE = 2 * K_BYTES;
    static constexpr int KSC = 2 * TILE, INFO = KSC + 2 * 64 * 4, BYTES = INFO + 2 * 16;
};

template <int HD, int NWV, int NS>
__global__ void __launch_bounds__(64 * NWV, 2)
attention_q8_rows_kernel(const bf16_t* __restrict__ q, bf16_t* __restrict__ out, float* __restrict__ part, Q8View v, int n_q, int window, int sinks,
                         float scale_log2, int chunk, int splits, int tiles) {
    constexpr int ROWS = 32 * NWV, HALF = 32 * NWV, CPT = 64 * HD / HALF, VC = CPT / 8;   // threads that stage one half; codes and columns of each
    constexpr int QC = HD / 32, HB = HD / 16;
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
    const int v_oct = st / (HD / VC), v_col = st % (HD / VC) * VC;                            // values: VC columns of eight keys
    const int v_key = (v_oct >> 2) * 32 + (v_oct & 3) * 4;                                  // ... v_key + 0..3 and + 16..19

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
        float m[2] = {-1e30f, -1e30f}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < HB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        int e_acc = 0;

        // ---- a tile's way from memory through registers into LDS
        unsigned raw[CPT / 4];
        float sc8[2][NS], sc1 = 0.f;
        bool bad = false;
        int phys = 0, off = 0, e_now = 0, e_most = -1000;
        auto look_up = [&](int i) {
            const int key0 = ks.at(i) * 64, pg = key0 / v.page_tokens;
            off = key0 - pg * v.page_tokens;
            phys = v.table[size_t(s) * v.pages_per_seq + pg];
        };
        auto load = [&] {
            bad = phys < 0 || phys >= v.n_phys;
            const unsigned char* page = v.base + size_t(bad ? 0 : phys) * v.page_bytes + (keys_half ? 0 : v.half_bytes);
            const unsigned char* codes = page + (size_t(g) * v.page_tokens + off) * HD;
            const float* scales = (const float*)(page + v.scales_off);
            const int at = g * v.page_tokens + off;
            if (keys_half) {
#pragma unroll
                for (int c = 0; c < CPT / 16; ++c) *(uint4*)&raw[4 * c] = *(const uint4*)(codes + k_key * HD + k_at + 16 * c);
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const unsigned char* p = codes + (v_key + (t < 4 ? t : t + 12)) * HD + v_col;
                    if constexpr (VC == 8) *(uint2*)&raw[2 * t] = *(const uint2*)p;
                    else if constexpr (VC == 4) raw[t] = *(const unsigned*)p;
                    else raw[t / 2] = t & 1 ? raw[t / 2] | unsigned(*(const unsigned short*)p) << 16 : *(const unsigned short*)p;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (NS == 4) *(float4*)sc8[h] = *(const float4*)(scales + at + v_key + 16 * h);
                    else sc8[h][0] = scales[(at + v_key + 16 * h) >> v.scale_shift];
                }
            }
            sc1 = scales[(at + lane) >> (NS == 4 ? 0 : v.scale_shift)];
        };
        auto stage = [&](int i, int buf) {
            unsigned char* base = lds + buf * L::TILE;
            const int key0 = ks.at(i) * 64;
            if (keys_half) {
#pragma unroll
                for (int c = 0; c < CPT / 8; ++c) {
                    const int piece = k_at / 8 + c;
                    *(bf16x8*)(base + k_key * (HD * 2) + ((piece ^ (k_key & 7)) << 4)) = codes8(raw[2 * c], raw[2 * c + 1]);
                }
                if (wave == 0) ((float*)(lds + L::KSC))[buf * 64 + lane] = bad ? __uint_as_float(0x7fc00000u) : sc1 * scale_log2;
            } else {
                auto seen = [&](int key) { return key <= pos_hi && (window <= 0 || key > pos_lo - window || key < sinks); };
                const bool mine = seen(key0 + lane), fine = fabsf(sc1) <= FLT_MAX;
                float top = mine && fine ? sc1 : 0.f;
                const unsigned long long mask = __builtin_amdgcn_ballot_w64(mine && !fine);
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
                top = max4(top);
                const unsigned bits = __builtin_amdgcn_readfirstlane(__float_as_uint(top));
                if (bits) {
                    const int e = int(bits >> 23) - 127;
                    e_most = max(e_most, e);
                    if (e > e_now + 3 || e < e_now - 3) e_now = max(e, e_most - 80);
                }
                if (wave == NWV / 2 && lane == 0) {
                    int* info = (int*)(lds + L::INFO + buf * 16);
                    info[0] = e_now; info[2] = int(unsigned(mask)); info[3] = int(unsigned(mask >> 32));
                }
                const float unit = ldexpf(1.f, -e_now);
                float f[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float x = sc8[t / 4][NS == 4 ? t & 3 : 0];
                    f[t] = seen(key0 + v_key + (t < 4 ? t : t + 12)) && fabsf(x) <= FLT_MAX ? x * unit : 0.f;
                }
#pragma unroll
                for (int j = 0; j < VC; ++j) {
                    auto val = [&](int t) {
                        const unsigned w = VC == 8 ? raw[2 * t + j / 4] : VC == 4 ? raw[t] : raw[t / 2];
                        return code(w, VC == 2 ? 2 * (t & 1) + j : j & 3) * f[t];
                    };
                    const uint4 x = {pack_half(val(0), val(1)), pack_half(val(2), val(3)), pack_half(val(4), val(5)), pack_half(val(6), val(7))};
                    const int row = v_col + j;
                    *(uint4*)(base + L::K_BYTES + row * 128 + ((v_oct ^ ((row ^ (row >> 3)) & 7)) << 4)) = x;
                }
            }
        };
        // ---- a tile's products
        auto work = [&](int i, int buf) {
            const int key0 = ks.at(i) * 64;
            if (key0 > w_hi) return;                                                        // nothing for this wave
            const bool edge = key0 + 63 > w_lo || w1 - w0 < 31 || (window > 0 && key0 <= w_hi - window && key0 + 63 >= sinks);
            const unsigned char* kb = lds + buf * L::TILE;
            const unsigned char* vb = kb + L::K_BYTES;
            const float* ksc = (const float*)(lds + L::KSC) + buf * 64;
            const int4 info = *(const int4*)(lds + L::INFO + buf * 16);
            f32x4 sc[4][2];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
#pragma unroll
                for (int r = 0; r < 2; ++r) sc[h][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    const bf16x8 kf = *(const bf16x8*)(kb + (16 * h + n16) * (HD * 2) + (((c * 4 + g4) ^ (n16 & 7)) << 4));
#pragma unroll
                    for (int r = 0; r < 2; ++r) sc[h][r] = mfma16(kf, qf[r][c], sc[h][r]);
                }
            }
            const int e_tile = __builtin_amdgcn_readfirstlane(info.x);
            if (e_tile != e_acc) {
                const float f = ldexpf(1.f, max(e_acc - e_tile, -126));
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int j = 0; j < HB; ++j) acc[r][j] *= f;
                e_acc = e_tile;
            }
            f16x8 wf[2][2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float top = -INFINITY;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float4 k4 = *(const float4*)(ksc + 16 * h + 4 * g4);
                    sc[h][r][0] *= k4.x; sc[h][r][1] *= k4.y; sc[h][r][2] *= k4.z; sc[h][r][3] *= k4.w;
                    if (edge)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + 16 * h + 4 * g4 + e;
                            const bool seen = key <= pos[r] && (window <= 0 || key > pos[r] - window || key < sinks);
                            sc[h][r][e] = seen ? sc[h][r][e] : -INFINITY;
                        }
                    top = fmaxf(fmaxf(top, fmaxf(sc[h][r][0], sc[h][r][1])), fmaxf(sc[h][r][2], sc[h][r][3]));
                }
                if (__builtin_amdgcn_ballot_w64(top > m[r] + W_TOP)) {
                    top = max4(top);
                    const float to = top > m[r] + W_TOP ? top - W_FIRST : m[r];
                    const float f = __builtin_amdgcn_exp2f(m[r] - to);
                    l[r] *= f;
#pragma unroll
                    for (int j = 0; j < HB; ++j) acc[r][j] *= f;
                    m[r] = to;
                }
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[h][r][e] = __builtin_amdgcn_exp2f(sc[h][r][e] - m[r]);
                        l[r] += sc[h][r][e];
                    }
                if (info.z | info.w) {      // values that are not finite
                    const unsigned long long mask = unsigned(info.z) | (unsigned long long)unsigned(info.w) << 32;
#pragma unroll
                    for (int h = 0; h < 4; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int k = 16 * h + 4 * g4 + e, key = key0 + k;
                            const bool seen = key <= pos[r] && (window <= 0 || key > pos[r] - window || key < sinks);
                            if (seen && (mask >> k & 1)) l[r] = __uint_as_float(0x7fc00000u);
                        }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint4 x = {pack_half(sc[2 * c][r][0], sc[2 * c][r][1]), pack_half(sc[2 * c][r][2], sc[2 * c][r][3]),
                                     pack_half(sc[2 * c + 1][r][0], sc[2 * c + 1][r][1]), pack_half(sc[2 * c + 1][r][2], sc[2 * c + 1][r][3])};
                    wf[r][c] = __builtin_bit_cast(f16x8, x);
                }
            }
#pragma unroll
            for (int j = 0; j < HB; ++j)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int row = 16 * j + n16;
                    const f16x8 vf = *(const f16x8*)(vb + row * 128 + (((c * 4 + g4) ^ ((row ^ (row >> 3)) & 7)) << 4));
#pragma unroll
                    for (int r = 0; r < 2; ++r) acc[r][j] = mfma16h(vf, wf[r][c], acc[r][j]);
                }
        };
        if (c0 < c1) {
            look_up(c0);
            load();
            stage(c0, 0);
            if (c0 + 1 < c1) { look_up(c0 + 1); load(); }
            __syncthreads();
            for (int i = c0; i < c1; ++i) {
                const int buf = (i - c0) & 1;
                if (i + 2 < c1) look_up(i + 2);
                if (i + 1 < c1) stage(i + 1, buf ^ 1);
                if (i + 2 < c1) load();
                work(i, buf);
                __syncthreads();
            }
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
                if (g4 == 0) { d[HD] = m[r]; d[HD + 1] = sum; }
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
    const int tile = std::max(16, 1 << v.scale_shift), tiles = std::min((max_rows + tile - 1) / tile + 1, std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv)));
    const size_t lds = size_t(tile) * (HD / 2) * sizeof(double2) + (2 * tile + 2) * 4;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)append_q8_kernel<T, HD>, hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((append_q8_kernel<T, HD>), dim3(unsigned(size_t(v.n_seqs) * tiles * v.n_kv)), dim3(256), lds, st, qkv, q, values, v, rope, n_q, tile, tiles);
    return hipGetLastError();
}

// How a launch divides the keys: `chunk` steps of `width` keys to a workgroup, at most `splits` ranges.
struct KeyRanges { int tiles, chunk, splits; int64_t groups; };
KeyRanges key_ranges(const Q8View& v, int n_q, int rows_per_tile, int width, int max_rows, int max_len, int window, int sinks, int least, int most, int64_t want,
                     const AttnWs& ws) {
    KeyRanges k;
    const int G = n_q / v.n_kv;
    k.tiles = int(std::min<int64_t>((int64_t(max_rows) * G + rows_per_tile - 1) / rows_per_tile, std::max(1, MOST_GROUPS / (v.n_seqs * v.n_kv))));
    const int64_t seen = window > 0 ? std::min<int64_t>(max_len, int64_t(window) + sinks + rows_per_tile / G + 2 * width) : max_len;
    const int64_t steps = seen / width + 1;
    k.groups = int64_t(v.n_seqs) * v.n_kv * k.tiles;
    int64_t chunk = std::min<int64_t>(std::max<int64_t>(least, (steps * k.groups + want - 1) / want), most);
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
    const KeyRanges k = key_ranges(v, n_q, 16 * NB, 32, max_rows, max_len, window, sinks, 4, 32, 2048, ws);
    hipLaunchKernelGGL((attention_q8_kernel<T, HD, NB, NS>), dim3(unsigned(k.groups * k.splits)), dim3(256), 0, st, q, out, ws.part, v, n_q, window, sinks,
                       scale, k.chunk, k.splits, k.tiles);
    return merge_q8(v, n_q, k, ws, out, st);
}

template <int HD, int NWV, int NS>
hipError_t attention_q8_rows(const bf16_t* q, bf16_t* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks, float scale, const AttnWs& ws,
                             hipStream_t st) {
    const KeyRanges k = key_ranges(v, n_q, 32 * NWV, 64, max_rows, max_len, window, sinks, 4, 1 << 20, 256, ws);
    constexpr int LDS = RowsLds<HD>::BYTES;
    static bool set = false;
    if (!set) {
        const hipError_t e = hipFuncSetAttribute((const void*)attention_q8_rows_kernel<HD, NWV, NS>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
        set = true;
    }
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
    const float scale = 1.44269504088896340736f / std::sqrt(float(v.head_dim));
    auto go = [&](auto hd, auto ns) {
        constexpr int HD = decltype(hd)::value, NS = decltype(ns)::value;
        if (dtype == CAKE_F32) return attention_q8<float, HD, 1, NS>((const float*)q, (float*)out, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        const bf16_t* qb = (const bf16_t*)q;
        bf16_t* ob = (bf16_t*)out;
        if (rows <= 16) return attention_q8<bf16_t, HD, 1, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        if (rows <= 32) return attention_q8<bf16_t, HD, 2, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        if (rows <= 128) return attention_q8_rows<HD, 4, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
        return attention_q8_rows<HD, 8, NS>(qb, ob, v, n_q, max_rows, max_len, window, sinks, scale, ws, st);
    };
    const std::integral_constant<int, 128> hd128{};
    const std::integral_constant<int, 64> hd64{};
    const std::integral_constant<int, 4> each{};     // a scale per token: four neighbours' at once
    const std::integral_constant<int, 1> shared{};   // four tokens or more share one
    if (v.scale_shift == 0) return v.head_dim == 128 ? go(hd128, each) : go(hd64, each);
    return v.head_dim == 128 ? go(hd128, shared) : go(hd64, shared);
}

}  // namespace cake
