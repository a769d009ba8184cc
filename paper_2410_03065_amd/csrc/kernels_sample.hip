// The next token of each row of logits: temperature, top-k, top-p, min-p, and a given random number.
//
// With z_i = (l_i - l_max) / T the weight of token i is exp(z_i), held as a whole number w_i = rint(2^44 exp(z_i)), computed
// in 64 bits (full rate on this chip).  Whole numbers add up to the same sum in any order, so nothing depends on how a row is
// divided or on the order of atomics; 2^19 tokens fit 64 bits, and an error of 2^-45 moves a border between tokens by less
// than the random number's own step.  Tokens rank by logit, equal ones by id; what each filter keeps is the ranking's front,
// so a row's kept set is a threshold on (logit, id).  The token is the first kept one in the order of ids whose running sum
// exceeds u times the total.
//
// A row's steps: its maximum; then, where top-k or top-p ask for it, counts and weights over 1024 bins of z; then the tokens of
// the bin that a filter ends in, or of all bins up to it where those are few; a workgroup ends the row on that list.  Bins of equal
// width in z spread logits evenly, where the leading bits of floating numbers would crowd them into a few; only a bin with more than
// LIST tokens is divided further by its keys' digits.  Rows without those filters skip the bins.
// Up to 32768 logits one workgroup holds a row in its registers and takes all steps in one launch: one row of 32000 with all
// filters 21 us, 256 rows of 32003 with none 20 (four kernels over slices: 30 and 39), bound by the latency of a workgroup's
// steps and by the 64-bit weights (9 of 20).  Longer rows are read in slices by many workgroups, a kernel a step (the bytes are in
// the caches from the second on): 64 rows of 128256 take 8 + 19 + 16 + 16 us, bound by the bins' LDS atomics and the end's sorts.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.hpp"

namespace cake {
namespace {

typedef unsigned long long u64;
constexpr int BINS = 1024, LIST = 4096, SHORT = 512, SLICES = 64;
constexpr double ONE = 17592186044416.0;          // 2^44, the weight of the likeliest token
constexpr double LEAST_OCTAVE = 45.0, BINS_PER_OCTAVE = 22.0;   // what has a weight fills 990 of the 1024 bins

// What the bins say.  Filters end in a bin: top-k in k_bin (none: BINS), top-p, if it alone counts, in p_bin.
enum Mode {
    WHOLE,     // no filter cuts anything
    FRONT,     // the list holds all bins up to `last`, everything that can be kept: SHORT tokens or fewer
    BIN,       // the list holds bin `last` alone
    DIGITS     // bin `last` has more than LIST tokens
};
struct Plan {
    Mode mode;
    bool by_count;            // `last` is where top-k ends (else top-p)
    int last;
    unsigned before;          // tokens of the bins before it
    u64 mass_before, total;   // weight of the bins before it; of all
};
struct Row {
    u64 mass[BINS];
    unsigned count[BINS];
    u64 slice_best[SLICES], part_mass[SLICES * 4];
    unsigned list_n, pad;
    Plan plan;
    u64 list[LIST];
};
static_assert(sizeof(Row) == SAMPLE_ROW_BYTES);

struct Args {
    const float* logits; int64_t stride; int rows_n, vocab, slices, slice_len;
    const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p; const float* u;
    int32_t* tokens; float* logprobs; Row* rows;
};

// Workgroups go round the eight XCDs; their numbers go to runs of neighbours on each, so that a row's slices share one L2 with their
// sums and, from the second kernel on, their logits.  The grid: n rounded up to 8.
__device__ __forceinline__ int xcd_order(int n) { return int(blockIdx.x & 7) * ((n + 7) / 8) + int(blockIdx.x >> 3); }
inline unsigned xcd_grid(int n) { return unsigned((n + 7) / 8 * 8); }

// Float bits that order like the numbers; 0 for what can never be chosen (NaN).  -0 counts as 0.
__device__ __forceinline__ unsigned order(float l) {
    const unsigned b = __float_as_uint(l + 0.0f);
    return l != l ? 0u : b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unorder(unsigned k) { return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k); }
// (logit, id): larger is earlier in the ranking
__device__ __forceinline__ u64 rank_key(float l, int id) { return u64(order(l)) << 32 | unsigned(~id); }

// A wave's 64-bit values through its row shifts and broadcasts: lanes without a source get 0.
template <int CTRL, int ROWS> __device__ __forceinline__ u64 moved(u64 v) {
    return u64(unsigned(__builtin_amdgcn_update_dpp(0, int(v >> 32), CTRL, ROWS, 0xf, true))) << 32 |
           unsigned(__builtin_amdgcn_update_dpp(0, int(v), CTRL, ROWS, 0xf, true));
}
template <typename F> __device__ __forceinline__ u64 wave_fold(u64 v, F f) {   // inclusive, lane by lane
    v = f(v, moved<0x111, 0xf>(v));   // row_shr:1, 2, 4, 8
    v = f(v, moved<0x112, 0xf>(v));
    v = f(v, moved<0x114, 0xf>(v));
    v = f(v, moved<0x118, 0xf>(v));
    v = f(v, moved<0x142, 0xa>(v));   // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    return f(v, moved<0x143, 0xc>(v));
}
__device__ __forceinline__ u64 last_lane(u64 v) {
    return u64(unsigned(__builtin_amdgcn_readlane(int(v >> 32), 63))) << 32 | unsigned(__builtin_amdgcn_readlane(int(v), 63));
}
__device__ __forceinline__ u64 wave_scan(u64 v) { return wave_fold(v, [](u64 a, u64 b) { return a + b; }); }
__device__ __forceinline__ u64 wave_sum(u64 v) { return last_lane(wave_scan(v)); }
__device__ __forceinline__ u64 wave_max(u64 v) { return last_lane(wave_fold(v, [](u64 a, u64 b) { return a > b ? a : b; })); }

struct Params {
    float top;          // the row's largest logit
    double octaves;     // log2(e) / T
    float bins_scale, sure;   // logits to bins; bins up to `sure` certainly weigh something
    int best, k;        // the likeliest token (-1: every logit is -infinity or NaN); top-k, 0: off
    double p;           // >= 1: off
    u64 least;          // least weight that is kept
    bool greedy, bins;
};
__device__ __forceinline__ Params params(const Args& a, int row, u64 best) {
    Params r;
    r.top = unorder(unsigned(best >> 32));
    r.best = unsigned(best >> 32) <= order(-INFINITY) ? -1 : int(~unsigned(best));
    const float t = a.temperature ? a.temperature[row] : 1.f;
    r.greedy = !(t > 0.f) || r.best < 0;
    r.octaves = 1.4426950408889634074 / double(t);
    const double scale = 2.0 * r.octaves * BINS_PER_OCTAVE;
    r.bins_scale = float(fmin(scale, 3e38));
    r.sure = scale < 3e38 ? float(LEAST_OCTAVE * BINS_PER_OCTAVE) - 1.f : -1.f;
    r.k = a.top_k ? a.top_k[row] : 0;
    if (r.k < 0 || r.k >= a.vocab) r.k = 0;
    const float p = a.top_p ? a.top_p[row] : 1.f, low = a.min_p ? a.min_p[row] : 0.f;
    r.p = p < 1.f ? double(p) : 1.0;
    r.least = low > 0.f ? max(u64(1), u64(rint(fmin(double(low), 1.0) * ONE))) : 1;
    r.bins = !r.greedy && (r.k > 0 || r.p < 1.0);
    return r;
}
__device__ __forceinline__ Params params(const Args& a, int row) {
    const int lane = threadIdx.x & 63;
    return params(a, row, wave_max(lane < a.slices ? a.rows[row].slice_best[lane] : 0));
}

// z of a token in octaves below the likeliest one's (0 or less); NaN where it can never be chosen.
__device__ __forceinline__ double octaves(float l, const Params& r) {
    const double y = (double(l) - double(r.top)) * r.octaves;
    return l == r.top ? 0.0 : y;                    // also where both are infinite
}
__device__ __forceinline__ bool weighs(double y) { return y > -LEAST_OCTAVE; }
// Its weight where it weighs.  2^f on |f| <= 1/2 by the polynomial that meets it at the eleven Chebyshev points: 3e-16 off, 1 at
// f = 0.  Adding a number with a unit of 1 in its last place rounds to a whole number and leaves it in the low bits.
__device__ __forceinline__ u64 weight_at(double y) {
    const double whole = y + 6755399441055744.0;       // 1.5 * 2^52
    const double f = y - (whole - 6755399441055744.0);
    double p = 7.072585949269223e-09;
    p = fma(p, f, 1.0208690299958306e-07); p = fma(p, f, 1.321544258792169e-06); p = fma(p, f, 1.5252657260200837e-05);
    p = fma(p, f, 0.0001540353044173605); p = fma(p, f, 0.0013333558230164974); p = fma(p, f, 0.009618129107606888);
    p = fma(p, f, 0.05550410866444772); p = fma(p, f, 0.24022650695910097); p = fma(p, f, 0.69314718055995); p = fma(p, f, 1.0);
    const u64 scaled = u64(__double_as_longlong(p)) + (u64(unsigned(__double_as_longlong(whole)) + 44u) << 52);   // times 2^(n + 44)
    return u64(__double_as_longlong(__longlong_as_double(scaled) + 4503599627370496.0)) & 0xfffffffffffffull;
}
// 1 or more where it weighs
__device__ __forceinline__ u64 weight(float l, const Params& r) {
    const double y = octaves(l, r);
    return weighs(y) ? max(u64(1), weight_at(y)) : 0;
}
// 0 below the least weight that is kept
__device__ __forceinline__ u64 kept_weight(float l, const Params& r) {
    const double y = octaves(l, r);
    const u64 w = weight_at(y);
    return weighs(y) && w >= r.least ? w : 0;
}

// The elements of a range, eight loads a thread at a time, of NT threads (64: each wave has a range of its own): f(element, its number).
template <int NT, typename F> __device__ __forceinline__ void each(const float* l, int lo, int hi, F f) {
    for (int i = lo + int(threadIdx.x & (NT - 1)); i < hi; i += 8 * NT) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = l[min(i + k * NT, hi - 1)];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k * NT < hi) f(x[k], i + k * NT);
    }
}

// Where a token lies among the bins, in 32 bits: which bin it falls into is free as long as lower logits fall no earlier.  Whether
// it weighs anything is not, so it is decided in 64 bits where 32 leave it open.  No bin (infinity) for what weighs nothing.
__device__ __forceinline__ float place_of(float l, const Params& r) {
    const float t = l == r.top ? 0.f : (0.5f * r.top - 0.5f * l) * r.bins_scale;      // halves: their difference is finite
    if (t < r.sure) return t;
    return t < r.sure + 2.f || (r.sure < 0.f && t < BINS) ? (weighs(octaves(l, r)) ? t : INFINITY) : INFINITY;
}
__device__ __forceinline__ int bin_of(float t) { return int(t); }

// Exclusive sums over the workgroup's threads; s: a word per wave.  All threads call it.
template <int NT> __device__ __forceinline__ u64 block_scan(u64 v, u64* s, u64* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 in = wave_scan(v);
    __syncthreads();
    if (lane == 63) s[wave] = in;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) { if (w < wave) before += s[w]; all += s[w]; }
    *total = all;
    return before + in - v;
}

// A slice is dealt to its workgroup's four waves in parts: where this thread's (or with next: the one after it) begins.
__device__ __forceinline__ int part_begin(const Args& a, int slice, int next = 0) {
    const int lo = slice * a.slice_len, hi = min(a.vocab, lo + a.slice_len);
    return min(hi, lo + (int(threadIdx.x >> 6) + next) * ((a.slice_len + 3) / 4));
}

// ---- the largest logit of each slice; the rows' sums cleared
__global__ void __launch_bounds__(256) sample_max_kernel(Args a) {
    const int at = xcd_order(a.rows_n * a.slices), row = at / a.slices, slice = at % a.slices;
    if (row >= a.rows_n) return;
    Row& r = a.rows[row];
    for (int i = slice * 256 + threadIdx.x; i < BINS; i += a.slices * 256) { r.mass[i] = 0; r.count[i] = 0; }
    if (slice == 0 && threadIdx.x == 0) r.list_n = 0;
    const float* l = a.logits + row * a.stride;
    const int lo = slice * a.slice_len, hi = min(a.vocab, lo + a.slice_len);
    u64 best = 0;
    each<256>(l, lo, hi, [&](float x, int i) { best = max(best, rank_key(x, i)); });
    best = wave_max(best);
    __shared__ u64 s[4];
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = best;
    __syncthreads();
    if (threadIdx.x == 0) r.slice_best[slice] = max(max(s[0], s[1]), max(s[2], s[3]));
}

// Finds the bin in which a running count (by_count) or weight reaches `need`: sums before < need <= sums through it.
template <int NT> __device__ __forceinline__ bool find_bin(const u64* mass, const unsigned* count, bool by_count, double need, u64* s, Plan* shared, Plan* out) {
    constexpr int PER = BINS / NT;
    u64 m = 0, c = 0, mass_all, count_all;
#pragma unroll
    for (int i = 0; i < PER; ++i) { m += mass[threadIdx.x * PER + i]; c += count[threadIdx.x * PER + i]; }
    u64 mb = block_scan<NT>(m, s, &mass_all), cb = block_scan<NT>(c, s, &count_all);
    if (threadIdx.x == 0) { shared->last = BINS; shared->total = mass_all; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const u64 mi = mass[threadIdx.x * PER + i], ci = count[threadIdx.x * PER + i];
        const double b = by_count ? double(cb) : double(mb), e = by_count ? double(cb + ci) : double(mb + mi);
        if (b < need && need <= e) { shared->last = threadIdx.x * PER + i; shared->before = unsigned(cb); shared->mass_before = mb; }
        mb += mi; cb += ci;
    }
    __syncthreads();
    *out = *shared;
    __syncthreads();
    return out->last < BINS;
}
template <int NT> __device__ __forceinline__ Plan plan(const u64* mass, const unsigned* count, const Params& p, u64* s, Plan* shared) {
    Plan o;
    o.by_count = p.k > 0 && find_bin<NT>(mass, count, true, double(p.k), s, shared, &o);
    bool cut = o.by_count;
    if (!cut && p.p < 1.0) {
        u64 total;
        u64 m = 0;
        for (int i = threadIdx.x; i < BINS; i += NT) m += mass[i];
        block_scan<NT>(m, s, &total);
        cut = find_bin<NT>(mass, count, false, fmax(p.p * double(total), 1.0), s, shared, &o);
        o.by_count = false;
    }
    if (!cut) { o.mode = WHOLE; o.last = BINS; return o; }
    const unsigned in = count[o.last];
    o.mode = o.before + in <= SHORT ? FRONT : in <= LIST ? BIN : DIGITS;
    return o;
}

// ---- counts and weights by bin, or the slice's weight where no filter needs bins
__global__ void __launch_bounds__(256) sample_bins_kernel(Args a) {
    __shared__ u64 mass[BINS];
    __shared__ unsigned count[BINS];
    const int at = xcd_order(a.rows_n * a.slices), row = at / a.slices, slice = at % a.slices;
    if (row >= a.rows_n) return;
    const Params p = params(a, row);
    if (p.greedy) return;
    Row& r = a.rows[row];
    const float* l = a.logits + row * a.stride;
    const int lo = slice * a.slice_len, hi = min(a.vocab, lo + a.slice_len);
    if (!p.bins) {
        u64 sum = 0;
        each<64>(l, part_begin(a, slice), part_begin(a, slice, 1), [&](float x, int) { sum += kept_weight(x, p); });
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) r.part_mass[slice * 4 + (threadIdx.x >> 6)] = sum;
        return;
    }
    for (int i = threadIdx.x; i < BINS; i += 256) { mass[i] = 0; count[i] = 0; }
    __syncthreads();
    const bool masses = p.p < 1.0;     // top-k alone counts
    each<256>(l, lo, hi, [&](float x, int) {
        const float t = place_of(x, p);
        if (!(t < BINS)) return;
        if (masses) atomicAdd(&mass[bin_of(t)], weight(x, p));
        atomicAdd(&count[bin_of(t)], 1u);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += 256)
        if (count[i]) { if (masses) atomicAdd(&r.mass[i], mass[i]); atomicAdd(&r.count[i], count[i]); }
}

// ---- the tokens that the end of the row is decided on, and the weight of those that are certainly kept
__global__ void __launch_bounds__(256) sample_gather_kernel(Args a) {
    __shared__ u64 s[4], list[LIST];       // with a plan of a list no slice has more
    __shared__ unsigned listed, base;
    __shared__ Plan shared;
    const int at = xcd_order(a.rows_n * a.slices), row = at / a.slices, slice = at % a.slices;
    if (row >= a.rows_n) return;
    const Params p = params(a, row);
    if (!p.bins) return;
    Row& r = a.rows[row];
    if (threadIdx.x == 0) listed = 0;
    const Plan o = plan<256>(r.mass, r.count, p, s, &shared);
    if (slice == 0 && threadIdx.x == 0) r.plan = o;
    if (o.mode == DIGITS) return;
    const float* l = a.logits + row * a.stride;
    const float from = o.mode == FRONT ? 0.f : float(o.last), end = float(o.last + 1);      // WHOLE: all of it
    u64 sum = 0;
    each<64>(l, part_begin(a, slice), part_begin(a, slice, 1), [&](float x, int i) {
        const float t = place_of(x, p);
        if (!(t < end)) return;
        if (t < from) {
            sum += kept_weight(x, p);
        } else {
            const unsigned n = atomicAdd(&listed, 1u);
            if (n < LIST) list[n] = rank_key(x, i);
        }
    });
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) r.part_mass[slice * 4 + (threadIdx.x >> 6)] = sum;
    // one of the device's atomics a workgroup: each takes a microsecond or more to return
    __syncthreads();
    const unsigned n = min(listed, unsigned(LIST));
    if (n == 0) return;
    if (threadIdx.x == 0) base = atomicAdd(&r.list_n, n);
    __syncthreads();
    for (unsigned i = threadIdx.x; i < n && base + i < LIST; i += 256) r.list[base + i] = list[i];
}

// ---- the row's token
// What the workgroup that ends a row holds.
template <int NT> struct Ends {
    u64 list[LIST], s[NT / 64], parts[SLICES * 4], digits[256], last_kept;
    unsigned count[256], pick, listed;
    Plan plan;
    int found, many_kept;
};

// The value of the lane whose number differs in bit J.
template <int J> __device__ __forceinline__ int crossed(int v) {
    if constexpr (J == 1) return __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);            // quads 1 0 3 2
    if constexpr (J == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);            // quads 2 3 0 1
    if constexpr (J == 4)                                                                            // l ^ 7, then ^ 3
        return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);
    if constexpr (J == 8) return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);           // rows turned by 8
    if constexpr (J >= 16) return __shfl_xor(v, J);
}
template <int J> __device__ __forceinline__ u64 crossed64(u64 v) { return u64(unsigned(crossed<J>(int(v >> 32)))) << 32 | unsigned(crossed<J>(int(v))); }

// Sorts s[0 .. n) from the largest to the smallest: a bitonic network on C values a thread, element c * NT + thread.  Elements closer
// than 64 lie in a wave and those NT or more apart in a thread; only the distances between go through LDS.
template <int NT, int C> __device__ __forceinline__ void sort_values(u64* s, int n, int up) {
    u64 v[C];
    const int t = threadIdx.x;
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = c * NT + t < n ? s[c * NT + t] : 0;
    auto keep = [&](int c, u64 other, int k, int j) {       // of two elements the larger goes to the lower place where the run falls
        const int i = c * NT + t;
        if ((v[c] < other) == (((i & k) == 0) == ((i & j) == 0))) v[c] = other;
    };
    auto cross = [&](auto j_, int k) {
        constexpr int J = decltype(j_)::value;
        if (J >= k) return;
#pragma unroll
        for (int c = 0; c < C; ++c) keep(c, crossed64<J>(v[c]), k, J);
    };
    for (int k = 2; k <= up; k <<= 1) {
        if constexpr (C > 1)
#pragma unroll
            for (int d = C / 2; d; d >>= 1)
                if (d * NT < k) {
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if (!(c & d)) { const u64 low = v[c], high = v[c + d]; keep(c, high, k, d * NT); keep(c + d, low, k, d * NT); }
                }
        for (int j = min(k, NT) >> 1; j >= 64; j >>= 1) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c) s[c * NT + t] = v[c];
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c) keep(c, s[c * NT + (t ^ j)], k, j);
        }
        cross(std::integral_constant<int, 32>(), k);
        cross(std::integral_constant<int, 16>(), k);
        cross(std::integral_constant<int, 8>(), k);
        cross(std::integral_constant<int, 4>(), k);
        cross(std::integral_constant<int, 2>(), k);
        cross(std::integral_constant<int, 1>(), k);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) s[c * NT + t] = v[c];
    __syncthreads();
}
template <int NT> __device__ __forceinline__ void sort_down(u64* s, int n) {
    int up = 2;
    while (up < n) up <<= 1;
    __syncthreads();
    if (up <= NT) sort_values<NT, 1>(s, n, up);
    else if (up == 2 * NT) sort_values<NT, 2>(s, n, up);
    else if (up == 4 * NT) sort_values<NT, 4>(s, n, up);
    else if constexpr (8 * NT <= LIST) sort_values<NT, 8>(s, n, up);
}

// The first id in [lo, hi) whose running sum of f exceeds `target`; the range's sum has to.  f(logit, id): a whole number.
template <int NT, typename F> __device__ __forceinline__ int first_past(const float* l, F f, int lo, int hi, u64 target, u64* s, int* found) {
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    while (hi - lo > 64) {
        const int seg = (hi - lo + NW - 1) / NW, b = lo + wave * seg;
        u64 sum = 0;
        each<64>(l, b, min(hi, b + seg), [&](float x, int i) { sum += f(x, i); });
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) s[wave] = sum;
        __syncthreads();
        int w = 0;
        for (; w < NW - 1 && target >= s[w]; ++w) target -= s[w];
        lo += w * seg;
        hi = min(hi, lo + seg);
    }
    __syncthreads();
    if (wave == 0) {
        const u64 v = lo + lane < hi ? f(l[lo + lane], lo + lane) : 0, in = wave_scan(v);
        if (in > target && in - v <= target) *found = lo + lane;
    }
    __syncthreads();
    return *found;
}

// The last kept rank key of bin `last` when `need` more tokens (by_count) or a running weight of `need` (starting at `mass`)
// are kept from it: digit by digit, the whole row read for each; *kept: the weight kept through it.
template <int NT> __device__ u64 by_digits(const float* l, int vocab, const Params& p, int last, bool by_count, double need, u64 mass, Ends<NT>& e, u64* kept) {
    unsigned prefix = 0;
    u64 count = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += NT) { e.digits[i] = 0; e.count[i] = 0; }
        __syncthreads();
        each<NT>(l, 0, vocab, [&](float x, int) {
            const float t = place_of(x, p);
            const unsigned k = order(x);
            if (!(t < BINS) || bin_of(t) != last || (shift < 24 && k >> (shift + 8) != prefix >> (shift + 8))) return;
            atomicAdd(&e.digits[k >> shift & 255], weight(x, p));
            atomicAdd(&e.count[k >> shift & 255], 1u);
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 m = mass, c = count;
            int d = 255;
            for (; d > 0; --d) {
                const double end = by_count ? double(c + e.count[d]) : double(m + e.digits[d]);
                if (e.count[d] && need <= end) break;
                m += e.digits[d]; c += e.count[d];
            }
            e.s[0] = m; e.s[1] = c; e.pick = unsigned(d);
        }
        __syncthreads();
        mass = e.s[0]; count = e.s[1];
        prefix |= e.pick << shift;
    }
    // equal logits: the first `ties` of them by id
    const u64 w = weight(unorder(prefix), p);
    u64 ties = by_count ? u64(need) - count : 1;
    if (!by_count)
        for (; double(mass + ties * w) < need; ++ties) {
            const double more = (need - double(mass + ties * w)) / double(w);     // many at once where many are missing
            if (more > 2.0) ties += u64(more) - 1;
        }
    *kept = mass + ties * w;
    __syncthreads();
    const int id = first_past<NT>(l, [&](float x, int) -> u64 { return order(x) == prefix; }, 0, vocab, ties - 1, e.s, &e.found);
    return u64(prefix) << 32 | unsigned(~id);
}

// Ends a row by its plan, its bins, the n tokens in e.list (FRONT, BIN) and e.parts, the weights of its parts without those tokens.
template <int NT> __device__ __forceinline__ void end_row(const Args& a, int row, const Params& p, const Plan& o, const u64* mass, const unsigned* count, int n,
                                                          Ends<NT>& e) {
    constexpr int NW = NT / 64;
    const float* l = a.logits + row * a.stride;
    const double u = fmin(fmax(double(a.u[row]), 0.0), 1.0);       // NaN counts as 0
    auto place = [&](u64 total) { return min(u64(u * double(total)), total - 1); };
    auto done = [&](int id, u64 total) {
        if (threadIdx.x != 0) return;
        a.tokens[row] = id;
        const double z = l[id] == p.top ? 0.0 : (double(l[id]) - double(p.top)) * p.octaves * 0.69314718055994530942;
        if (a.logprobs) a.logprobs[row] = float(z - log(double(total) / ONE));
    };
    auto weight_of_key = [&](u64 key) { return weight(unorder(unsigned(key >> 32)), p); };
    // the number of the list's first n tokens that are kept when a running weight starting at `mass` may not reach `need`
    // before a token; *kept: the weight through them
    auto ranks_before = [&](int n, u64 mass, double need, u64* kept) {
        u64 run = mass;
        if (threadIdx.x == 0) { e.last_kept = mass; e.many_kept = 0; }
        for (int b = 0; b < n; b += NT) {
            const int i = b + int(threadIdx.x);
            const u64 w = i < n ? weight_of_key(e.list[i]) : 0;
            u64 sum;
            const u64 before = run + block_scan<NT>(w, e.s, &sum);
            run += sum;
            // the kept are a front: its last one knows their weight
            if (i < n && double(before) < need && (i == n - 1 || !(double(before + w) < need))) { e.last_kept = before + w; e.many_kept = i + 1; }
        }
        __syncthreads();
        *kept = e.last_kept;
        const int many = e.many_kept;
        __syncthreads();
        return many;
    };
    const double none = 1e300;      // a weight that is never reached
    if (threadIdx.x == 0) e.found = p.best;

    u64 least_key = 0;              // kept: rank keys from here on
    bool have_parts = true;
    const int listed = n;
    if (o.mode == FRONT || o.mode == BIN) sort_down<NT>(e.list, n);
    if (o.mode == FRONT) {
        u64 kept;
        if (o.by_count) n = min(n, p.k);
        if (p.p < 1.0) {
            u64 all = o.total;
            if (o.by_count) ranks_before(n, 0, none, &all);
            n = ranks_before(n, 0, fmax(p.p * double(all), 1.0), &kept);
        }
        // by id: (id, logit) from the last to the first; below the least weight: nothing
        const int i = threadIdx.x;
        if (i < n) {
            const u64 k = e.list[i];
            e.list[i] = weight_of_key(k) >= p.least ? (k & 0xffffffffull) << 32 | k >> 32 : 0;        // ~id first: the largest is the first id
        }
        sort_down<NT>(e.list, n);
        const u64 k = i < n ? e.list[i] : 0, w = k ? weight(unorder(unsigned(k)), p) : 0;
        u64 total;
        const u64 before = block_scan<NT>(w, e.s, &total), target = place(total);
        if (w && before <= target && target < before + w) e.found = int(~unsigned(k >> 32));
        __syncthreads();
        done(e.found, total);
        return;
    }
    if (o.mode == BIN || o.mode == DIGITS) {
        u64 kept;
        if (o.mode == BIN) {
            if (o.by_count) {
                n = p.k - int(o.before);
                ranks_before(n, o.mass_before, none, &kept);
            } else {
                n = ranks_before(n, o.mass_before, fmax(p.p * double(o.total), 1.0), &kept);
            }
            least_key = e.list[n - 1];
        } else {
            const double need = o.by_count ? double(p.k) - double(o.before) : fmax(p.p * double(o.total), 1.0);
            least_key = by_digits<NT>(l, a.vocab, p, o.last, o.by_count, need, o.mass_before, e, &kept);
            have_parts = false;
        }
        if (o.by_count && p.p < 1.0) {      // top-p within the first k
            const double need = fmax(p.p * double(kept), 1.0);
            u64 got;
            if (need > double(o.mass_before)) {       // it ends in the same bin
                if (o.mode == BIN) {
                    n = ranks_before(n, o.mass_before, need, &got);
                    least_key = e.list[n - 1];
                } else {
                    least_key = max(least_key, by_digits<NT>(l, a.vocab, p, o.last, false, need, o.mass_before, e, &got));
                }
            } else {
                Plan q;
                find_bin<NT>(mass, count, false, need, e.s, &e.plan, &q);
                if (count[q.last] <= LIST) {
                    if (threadIdx.x == 0) e.listed = 0;
                    __syncthreads();
                    each<NT>(l, 0, a.vocab, [&](float x, int i) {
                        const float t = place_of(x, p);
                        if (t < BINS && bin_of(t) == q.last) e.list[atomicAdd(&e.listed, 1u)] = rank_key(x, i);
                    });
                    __syncthreads();
                    n = int(e.listed);
                    sort_down<NT>(e.list, n);
                    n = ranks_before(n, q.mass_before, need, &got);
                    least_key = e.list[n - 1];
                } else {
                    least_key = by_digits<NT>(l, a.vocab, p, q.last, false, need, q.mass_before, e, &got);
                }
                have_parts = false;
            }
        }
    }
    auto weight_of = [&](float x, int i) -> u64 {
        return rank_key(x, i) >= least_key ? kept_weight(x, p) : 0;
    };
    // the parts' weights: known but for the list's tokens, or summed here
    const int parts = a.slices * 4, part_len = (a.slice_len + 3) / 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto begin_of = [&](int i) { return min(min(a.vocab, (i / 4 + 1) * a.slice_len), i / 4 * a.slice_len + i % 4 * part_len); };
    auto end_of = [&](int i) { return min(min(a.vocab, (i / 4 + 1) * a.slice_len), i / 4 * a.slice_len + (i % 4 + 1) * part_len); };
    __syncthreads();
    if (!have_parts) {
        for (int i = wave; i < parts; i += NW) {
            u64 sum = 0;
            each<64>(l, begin_of(i), end_of(i), [&](float x, int j) { sum += weight_of(x, j); });
            sum = wave_sum(sum);
            if (lane == 0) e.parts[i] = sum;
        }
    } else if (o.mode == BIN) {
        for (int i = threadIdx.x; i < listed; i += NT) {
            const u64 k = e.list[i], w = kept_weight(unorder(unsigned(k >> 32)), p);
            const int id = int(~unsigned(k)), in = id % a.slice_len;
            if (k >= least_key && w) atomicAdd(&e.parts[id / a.slice_len * 4 + in / part_len], w);
        }
    }
    __syncthreads();
    // four parts a lane
    u64 own[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { own[i] = lane * 4 + i < parts ? e.parts[lane * 4 + i] : 0; mine += own[i]; }
    const u64 run = wave_scan(mine), total = last_lane(run);
    u64 target = place(total);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(run > target));
    target -= wave_sum(lane < at ? mine : 0);
    int part = at * 4;
    for (; part < at * 4 + 3 && target >= e.parts[part]; ++part) target -= e.parts[part];
    __syncthreads();
    const int id = first_past<NT>(l, weight_of, begin_of(part), end_of(part), target, e.s, &e.found);
    done(id, total);
}
__device__ __forceinline__ void end_greedy(const Args& a, int row, const Params& p) {
    if (threadIdx.x == 0) { a.tokens[row] = p.best; if (a.logprobs) a.logprobs[row] = p.best < 0 ? -INFINITY : 0.f; }
}

__global__ void __launch_bounds__(512) sample_pick_kernel(Args a) {
    constexpr int NT = 512;
    __shared__ Ends<NT> e;
    const int row = xcd_order(a.rows_n);
    if (row >= a.rows_n) return;
    const Params p = params(a, row);
    if (p.greedy) return end_greedy(a, row, p);
    Row& r = a.rows[row];
    const Plan o = p.bins ? r.plan : Plan{WHOLE, false, BINS, 0, 0, 0};
    const int n = o.mode == FRONT || o.mode == BIN ? min(int(r.list_n), LIST) : 0;
    for (int i = threadIdx.x; i < n; i += NT) e.list[i] = r.list[i];
    for (int i = threadIdx.x; i < a.slices * 4; i += NT) e.parts[i] = r.part_mass[i];
    end_row<NT>(a, row, p, o, r.mass, r.count, n, e);
}

// ---- a whole row in the registers of one workgroup: one launch and one reading, where the vocabulary is short enough
constexpr int HELD_NT = 1024, HELD = 32, HELD_MOST = HELD_NT * HELD;      // wave w has the ids from w * 2048 on, 64 side by side
__global__ void __launch_bounds__(HELD_NT) sample_row_kernel(Args a) {
    constexpr int NT = HELD_NT;
    __shared__ Ends<NT> e;
    __shared__ u64 mass[BINS];
    __shared__ unsigned count[BINS];
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave * 64 * HELD + lane;
    const float* l = a.logits + row * a.stride;
    float x[HELD];
#pragma unroll
    for (int k = 0; k < HELD; ++k) x[k] = l[min(first + k * 64, a.vocab - 1)];
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (first + k * 64 >= a.vocab) x[k] = __uint_as_float(0x7fc00000u);       // NaN: never chosen
    mass[threadIdx.x] = 0;
    count[threadIdx.x] = 0;
    if (threadIdx.x == 0) e.listed = 0;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < HELD; ++k) top = fmaxf(top, x[k]);
    int at = 0;
#pragma unroll
    for (int k = HELD - 1; k >= 0; --k) at = x[k] == top ? k : at;
    u64 best = wave_max(rank_key(top, first + at * 64));
    if (lane == 0) e.s[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) best = max(best, e.s[w]);
    const Params p = params(a, row, best);
    if (p.greedy) return end_greedy(a, row, p);
    Plan o = {WHOLE, false, BINS, 0, 0, 0};
    if (p.bins) {
        bool masses = false;
        if (p.k > 0) {                  // counts first: they are enough where top-k leaves few tokens
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                const float t = place_of(x[k], p);
                if (t < BINS) atomicAdd(&count[bin_of(t)], 1u);
            }
            __syncthreads();
            Params by_k = p;
            by_k.p = 1.0;
            o = plan<NT>(mass, count, by_k, e.s, &e.plan);
            masses = p.p < 1.0 && o.mode != FRONT;
        } else {
            masses = true;
        }
        if (masses) {
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                const float t = place_of(x[k], p);
                if (t < BINS) { atomicAdd(&mass[bin_of(t)], weight(x[k], p)); if (p.k == 0) atomicAdd(&count[bin_of(t)], 1u); }
            }
            __syncthreads();
            o = plan<NT>(mass, count, p, e.s, &e.plan);
        }
    }
    if (o.mode == WHOLE) {
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            u64 sum = 0;
#pragma unroll
            for (int k = part * 8; k < part * 8 + 8; ++k) sum += kept_weight(x[k], p);
            sum = wave_sum(sum);
            if (lane == 0) e.parts[wave * 4 + part] = sum;
        }
    } else if (o.mode == FRONT) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (place_of(x[k], p) < float(o.last + 1)) e.list[atomicAdd(&e.listed, 1u)] = rank_key(x[k], first + k * 64);
    } else if (o.mode == BIN) {
        const float from = float(o.last), end = float(o.last + 1);
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            u64 sum = 0;
#pragma unroll
            for (int k = part * 8; k < part * 8 + 8; ++k) {
                const float t = place_of(x[k], p);
                if (t < from) {
                    sum += kept_weight(x[k], p);
                } else if (t < end) {
                    e.list[atomicAdd(&e.listed, 1u)] = rank_key(x[k], first + k * 64);
                }
            }
            sum = wave_sum(sum);
            if (lane == 0) e.parts[wave * 4 + part] = sum;
        }
    }
    __syncthreads();
    end_row<NT>(a, row, p, o, mass, count, int(e.listed), e);
}
}  // namespace

hipError_t launch_sample(const SampleArgs& x, void* ws, size_t ws_bytes, hipStream_t st) {
    const int at_once = int(std::min<size_t>(size_t(x.rows), ws_bytes / sizeof(Row)));
    if (at_once < 1) return hipErrorInvalidValue;
    const bool held = x.vocab <= HELD_MOST;
    for (int r0 = 0; r0 < x.rows; r0 += held ? x.rows : at_once) {
        const int n = held ? x.rows : std::min(at_once, x.rows - r0);
        // slices of 2048 logits or more, about 1024 workgroups
        int slices = std::min(SLICES, std::min((x.vocab + 2047) / 2048, (1024 + n - 1) / n));
        int len = (x.vocab + slices - 1) / slices;
        slices = (x.vocab + len - 1) / len;
        if (held) { len = 64 * HELD; slices = (x.vocab + len - 1) / len; }
        const Args a = {x.logits + size_t(r0) * x.row_stride, x.row_stride, n, x.vocab, slices, len, x.temperature ? x.temperature + r0 : nullptr,
                        x.top_k ? x.top_k + r0 : nullptr, x.top_p ? x.top_p + r0 : nullptr, x.min_p ? x.min_p + r0 : nullptr, x.u + r0,
                        x.tokens + r0, x.logprobs ? x.logprobs + r0 : nullptr, (Row*)ws};
        if (held) {
            hipLaunchKernelGGL(sample_row_kernel, dim3(unsigned(n)), dim3(HELD_NT), 0, st, a);
        } else {
            hipLaunchKernelGGL(sample_max_kernel, dim3(xcd_grid(n * slices)), dim3(256), 0, st, a);
            hipLaunchKernelGGL(sample_bins_kernel, dim3(xcd_grid(n * slices)), dim3(256), 0, st, a);
            if (x.top_k || x.top_p) hipLaunchKernelGGL(sample_gather_kernel, dim3(xcd_grid(n * slices)), dim3(256), 0, st, a);
            hipLaunchKernelGGL(sample_pick_kernel, dim3(xcd_grid(n)), dim3(512), 0, st, a);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace cake
