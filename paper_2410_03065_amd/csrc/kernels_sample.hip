// The next token of each row of logits: temperature, top-k, top-p, min-p, and a given random number.
//
// With z_i = (l_i - l_max) / T the weight of token i is exp(z_i), held as a whole number w_i = rint(2^44 exp(z_i)), computed
// in 64 bits (full rate on this chip).  Whole numbers add up to the same sum in any order, so nothing depends on how a row is
// divided or on the order of atomics; 2^19 tokens fit 64 bits, and an error of 2^-45 moves a border between tokens by less
// than the random number's own step.  Tokens rank by logit, equal ones by id; what each filter keeps is the ranking's front,
// so a row's kept set is a threshold on (logit, id).  The token is the first kept one in the order of ids whose running sum
// exceeds u times the total.
//
// A row is read in slices by many workgroups (there may be one row): its maximum; then, where top-k or top-p ask for it, counts
// and weights over 1024 bins of z; then the tokens of the bin that a filter ends in, or of all bins up to it where those are
// few; one workgroup a row ends it on that list.  Bins of equal width in z spread logits evenly, where the leading bits of
// floating numbers would crowd them into a few; only a bin with more than LIST tokens is divided further by its keys' digits.
// Rows without those filters skip the bins.  Bound by reading the logits, from the second time on out of the caches.
#include <algorithm>
#include <cmath>

#include "kernels.hpp"

namespace cake {
namespace {

typedef unsigned long long u64;
constexpr int BINS = 1024, LIST = 4096, SHORT = 512, SLICES = 64;
constexpr double ONE = 17592186044416.0;          // 2^44, the weight of the likeliest token
constexpr double BINS_PER_OCTAVE = 22.0;          // 1024 bins over 46 octaves: everything that has a weight

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

struct Args {
    const float* logits; int64_t stride; int vocab, slices, slice_len;
    const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p; const float* u;
    int32_t* tokens; float* logprobs; Row* rows;
};

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
    int best, k;        // the likeliest token (-1: every logit is -infinity or NaN); top-k, 0: off
    double p;           // >= 1: off
    u64 least;          // least weight that is kept
    bool greedy, bins;
};
__device__ __forceinline__ Params params(const Args& a, int row) {
    Params r;
    const int lane = threadIdx.x & 63;
    const u64 best = wave_max(lane < a.slices ? a.rows[row].slice_best[lane] : 0);
    r.top = unorder(unsigned(best >> 32));
    r.best = unsigned(best >> 32) <= order(-INFINITY) ? -1 : int(~unsigned(best));
    const float t = a.temperature ? a.temperature[row] : 1.f;
    r.greedy = !(t > 0.f) || r.best < 0;
    r.octaves = 1.4426950408889634074 / double(t);
    r.k = a.top_k ? a.top_k[row] : 0;
    if (r.k < 0 || r.k >= a.vocab) r.k = 0;
    const float p = a.top_p ? a.top_p[row] : 1.f, low = a.min_p ? a.min_p[row] : 0.f;
    r.p = p < 1.f ? double(p) : 1.0;
    r.least = low > 0.f ? max(u64(1), u64(rint(fmin(double(low), 1.0) * ONE))) : 1;
    r.bins = !r.greedy && (r.k > 0 || r.p < 1.0);
    return r;
}

// z of a token in octaves below the likeliest one's (0 or less); NaN where it can never be chosen.
__device__ __forceinline__ double octaves(float l, const Params& r) {
    const double y = (double(l) - double(r.top)) * r.octaves;
    return l == r.top ? 0.0 : y;                    // also where both are infinite
}
__device__ __forceinline__ bool weighs(double y) { return y > -45.0; }
// Its weight, 1 or more where it weighs.  2^f on |f| <= 1/2 by its Taylor polynomial in f ln 2: the first term left out is
// 0.3466^12 / 12! = 6e-15.
__device__ __forceinline__ u64 weight_at(double y) {
    if (!weighs(y)) return 0;
    const double n = rint(y), f = (y - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800.0;
    p = fma(p, f, 1.0 / 3628800.0); p = fma(p, f, 1.0 / 362880.0); p = fma(p, f, 1.0 / 40320.0); p = fma(p, f, 1.0 / 5040.0);
    p = fma(p, f, 1.0 / 720.0); p = fma(p, f, 1.0 / 120.0); p = fma(p, f, 1.0 / 24.0); p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5); p = fma(p, f, 1.0); p = fma(p, f, 1.0);
    // adding 2^52 rounds to a whole number and leaves it in the low bits
    return max(u64(1), u64(__double_as_longlong(ldexp(p, int(n) + 44) + 4503599627370496.0)) & 0xfffffffffffffull);
}
__device__ __forceinline__ u64 weight(float l, const Params& r) { return weight_at(octaves(l, r)); }

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
__device__ __forceinline__ int bin_of(double y) { return min(BINS - 1, int(-y * BINS_PER_OCTAVE)); }

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
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
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

// ---- counts and weights by bin, or the slice's weight where no filter needs bins
__global__ void __launch_bounds__(256) sample_bins_kernel(Args a) {
    __shared__ u64 mass[BINS];
    __shared__ unsigned count[BINS];
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const Params p = params(a, row);
    if (p.greedy) return;
    Row& r = a.rows[row];
    const float* l = a.logits + row * a.stride;
    const int lo = slice * a.slice_len, hi = min(a.vocab, lo + a.slice_len);
    if (!p.bins) {
        u64 sum = 0;
        each<64>(l, part_begin(a, slice), part_begin(a, slice, 1), [&](float x, int) { const u64 w = weight(x, p); sum += w >= p.least ? w : 0; });
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) r.part_mass[slice * 4 + (threadIdx.x >> 6)] = sum;
        return;
    }
    for (int i = threadIdx.x; i < BINS; i += 256) { mass[i] = 0; count[i] = 0; }
    __syncthreads();
    const bool masses = p.p < 1.0;     // top-k alone counts
    each<256>(l, lo, hi, [&](float x, int) {
        const double y = octaves(x, p);
        if (!weighs(y)) return;
        if (masses) atomicAdd(&mass[bin_of(y)], weight_at(y));
        atomicAdd(&count[bin_of(y)], 1u);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += 256)
        if (count[i]) { if (masses) atomicAdd(&r.mass[i], mass[i]); atomicAdd(&r.count[i], count[i]); }
}

// Finds the bin in which a running count (by_count) or weight reaches `need`: sums before < need <= sums through it.
template <int NT> __device__ __forceinline__ bool find_bin(const Row& r, bool by_count, double need, u64* s, Plan* shared, Plan* out) {
    constexpr int PER = BINS / NT;
    u64 m = 0, c = 0, mass_all, count_all;
#pragma unroll
    for (int i = 0; i < PER; ++i) { m += r.mass[threadIdx.x * PER + i]; c += r.count[threadIdx.x * PER + i]; }
    u64 mb = block_scan<NT>(m, s, &mass_all), cb = block_scan<NT>(c, s, &count_all);
    if (threadIdx.x == 0) { shared->last = BINS; shared->total = mass_all; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const u64 mi = r.mass[threadIdx.x * PER + i], ci = r.count[threadIdx.x * PER + i];
        const double b = by_count ? double(cb) : double(mb), e = by_count ? double(cb + ci) : double(mb + mi);
        if (b < need && need <= e) { shared->last = threadIdx.x * PER + i; shared->before = unsigned(cb); shared->mass_before = mb; }
        mb += mi; cb += ci;
    }
    __syncthreads();
    *out = *shared;
    __syncthreads();
    return out->last < BINS;
}
template <int NT> __device__ __forceinline__ Plan plan(const Row& r, const Params& p, u64* s, Plan* shared) {
    Plan o;
    o.by_count = p.k > 0 && find_bin<NT>(r, true, double(p.k), s, shared, &o);
    bool cut = o.by_count;
    if (!cut && p.p < 1.0) {
        u64 total;
        u64 m = 0;
        for (int i = threadIdx.x; i < BINS; i += NT) m += r.mass[i];
        block_scan<NT>(m, s, &total);
        cut = find_bin<NT>(r, false, fmax(p.p * double(total), 1.0), s, shared, &o);
        o.by_count = false;
    }
    if (!cut) { o.mode = WHOLE; o.last = BINS; return o; }
    const unsigned in = r.count[o.last];
    o.mode = o.before + in <= SHORT ? FRONT : in <= LIST ? BIN : DIGITS;
    return o;
}

// ---- the tokens that the end of the row is decided on, and the weight of those that are certainly kept
__global__ void __launch_bounds__(256) sample_gather_kernel(Args a) {
    __shared__ u64 s[4];
    __shared__ Plan shared;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const Params p = params(a, row);
    if (!p.bins) return;
    Row& r = a.rows[row];
    const Plan o = plan<256>(r, p, s, &shared);
    if (slice == 0 && threadIdx.x == 0) r.plan = o;
    if (o.mode == DIGITS) return;
    const float* l = a.logits + row * a.stride;
    const int from = o.mode == FRONT ? 0 : o.last;
    u64 sum = 0;
    each<64>(l, part_begin(a, slice), part_begin(a, slice, 1), [&](float x, int i) {
        const double y = octaves(x, p);
        if (!weighs(y)) return;
        const int b = bin_of(y);
        if (b < from) {
            const u64 w = weight_at(y);
            sum += w >= p.least ? w : 0;
        } else if (b <= o.last && o.mode != WHOLE) {
            const unsigned at = atomicAdd(&r.list_n, 1u);
            if (at < LIST) r.list[at] = rank_key(x, i);
        }
    });
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) r.part_mass[slice * 4 + (threadIdx.x >> 6)] = sum;
}

// ---- the row's token
constexpr int NT = 512, NW = NT / 64;

// Sorts s[0 .. n) (n a power of two) from the largest to the smallest.  A wave's pairs of a stage of distance 64 or less lie in
// 128 elements of its own, and LDS serves a wave in order: only the wider stages need the others.
__device__ __forceinline__ void sort_down(u64* s, int n) {
    __syncthreads();
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j; j >>= 1) {
            if (j > 64 || (j == 64 && k > 128)) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int i = threadIdx.x; i < n / 2; i += NT) {
                const int x = (i / j) * 2 * j + i % j, y = x + j;
                const u64 p = s[x], q = s[y];
                if ((p < q) == ((x & k) == 0)) { s[x] = q; s[y] = p; }
            }
        }
    __syncthreads();
}

// The first id in [lo, hi) whose running sum of f exceeds `target`; the range's sum has to.  f(logit, id): a whole number.
template <typename F> __device__ __forceinline__ int first_past(const float* l, F f, int lo, int hi, u64 target, u64* s, int* found) {
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
__device__ u64 by_digits(const float* l, int vocab, const Params& p, int last, bool by_count, double need, u64 mass, u64* s, u64* d_mass, unsigned* d_count,
                         unsigned* pick, int* found, u64* kept) {
    unsigned prefix = 0;
    u64 count = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += NT) { d_mass[i] = 0; d_count[i] = 0; }
        __syncthreads();
        each<NT>(l, 0, vocab, [&](float x, int) {
            const double y = octaves(x, p);
            const unsigned k = order(x);
            if (!weighs(y) || bin_of(y) != last || (shift < 24 && k >> (shift + 8) != prefix >> (shift + 8))) return;
            atomicAdd(&d_mass[k >> shift & 255], weight_at(y));
            atomicAdd(&d_count[k >> shift & 255], 1u);
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 m = mass, c = count;
            int d = 255;
            for (; d > 0; --d) {
                const double end = by_count ? double(c + d_count[d]) : double(m + d_mass[d]);
                if (d_count[d] && need <= end) break;
                m += d_mass[d]; c += d_count[d];
            }
            s[0] = m; s[1] = c; *pick = unsigned(d);
        }
        __syncthreads();
        mass = s[0]; count = s[1];
        prefix |= *pick << shift;
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
    const int id = first_past(l, [&](float x, int) -> u64 { return order(x) == prefix; }, 0, vocab, ties - 1, s, found);
    return u64(prefix) << 32 | unsigned(~id);
}

__global__ void __launch_bounds__(NT) sample_pick_kernel(Args a) {
    __shared__ u64 list[LIST], s[NW], d_mass[SLICES * 4];     // d_mass: a digit's, then the parts'
    __shared__ unsigned d_count[256], pick, listed;
    __shared__ Plan shared;
    __shared__ int found, many_kept;
    __shared__ u64 last_kept;
    const int row = blockIdx.x;
    const Params p = params(a, row);
    if (p.greedy) {
        if (threadIdx.x == 0) { a.tokens[row] = p.best; if (a.logprobs) a.logprobs[row] = p.best < 0 ? -INFINITY : 0.f; }
        return;
    }
    if (threadIdx.x == 0) found = p.best;
    Row& r = a.rows[row];
    const float* l = a.logits + row * a.stride;
    const double u = fmin(fmax(double(a.u[row]), 0.0), 1.0);       // NaN counts as 0
    auto place = [&](u64 total) { return min(u64(u * double(total)), total - 1); };
    auto done = [&](int id, u64 total) {
        if (threadIdx.x != 0) return;
        a.tokens[row] = id;
        const double z = l[id] == p.top ? 0.0 : (double(l[id]) - double(p.top)) * p.octaves * 0.69314718055994530942;
        if (a.logprobs) a.logprobs[row] = float(z - log(double(total) / ONE));
    };
    // loads r.list (n tokens) into LDS, sorted from the first in the ranking
    auto take_list = [&](int n) {
        int up = 2;
        while (up < n) up <<= 1;
        for (int i = threadIdx.x; i < up; i += NT) list[i] = i < n ? r.list[i] : 0;
        sort_down(list, up);
    };
    // the number of the list's first n tokens that are kept when a running weight starting at `mass` may not reach `need`
    // before a token; *kept: the weight through them
    auto ranks_before = [&](int n, u64 mass, double need, u64* kept) {
        u64 run = mass;
        if (threadIdx.x == 0) { last_kept = mass; many_kept = 0; }
        for (int b = 0; b < n; b += NT) {
            const int i = b + int(threadIdx.x);
            const u64 w = i < n ? weight(unorder(unsigned(list[i] >> 32)), p) : 0;
            u64 sum;
            const u64 before = run + block_scan<NT>(w, s, &sum);
            run += sum;
            // the kept are a front: its last one knows their weight
            if (i < n && double(before) < need && (i == n - 1 || !(double(before + w) < need))) { last_kept = before + w; many_kept = i + 1; }
        }
        __syncthreads();
        *kept = last_kept;
        const int many = many_kept;
        __syncthreads();
        return many;
    };
    const double none = 1e300;      // a weight that is never reached

    u64 least_key = 0;              // kept: rank keys from here on
    bool have_slices = true;
    const Plan o = p.bins ? r.plan : Plan{WHOLE, false, BINS, 0, 0, 0};
    if (o.mode == FRONT) {
        int n = int(r.list_n);
        take_list(n);
        u64 kept;
        if (o.by_count) n = min(n, p.k);
        if (p.p < 1.0) {
            u64 all = o.total;
            if (o.by_count) ranks_before(n, 0, none, &all);
            n = ranks_before(n, 0, fmax(p.p * double(all), 1.0), &kept);
        }
        // by id: (id, logit) from the last to the first; below the least weight: nothing
        int up = 2;
        while (up < n) up <<= 1;
        __syncthreads();
        for (int i = threadIdx.x; i < up; i += NT) {
            const u64 k = i < n ? list[i] : 0;
            const bool in = i < n && weight(unorder(unsigned(k >> 32)), p) >= p.least;
            list[i] = in ? (k & 0xffffffffull) << 32 | k >> 32 : 0;        // ~id first: the largest is the first id
        }
        sort_down(list, up);
        u64 total = 0, run = 0;
        for (int pass = 0; pass < 2; ++pass) {
            const u64 target = pass ? place(total) : 0;
            for (int b = 0; b < up; b += NT) {
                const int i = b + int(threadIdx.x);
                const u64 k = i < up ? list[i] : 0, w = k ? weight(unorder(unsigned(k)), p) : 0;
                u64 sum;
                const u64 before = run + block_scan<NT>(w, s, &sum);
                if (pass && w && before <= target && target < before + w) found = int(~unsigned(k >> 32));
                run += sum;
            }
            if (!pass) { total = run; run = 0; }
        }
        __syncthreads();
        done(found, total);
        return;
    }
    if (o.mode == BIN || o.mode == DIGITS) {
        u64 kept;
        int n = 0;
        if (o.mode == BIN) {
            n = int(r.count[o.last]);
            take_list(n);
            if (o.by_count) {
                n = p.k - int(o.before);
                ranks_before(n, o.mass_before, none, &kept);
            } else {
                n = ranks_before(n, o.mass_before, fmax(p.p * double(o.total), 1.0), &kept);
            }
            least_key = list[n - 1];
        } else {
            const double need = o.by_count ? double(p.k) - double(o.before) : fmax(p.p * double(o.total), 1.0);
            least_key = by_digits(l, a.vocab, p, o.last, o.by_count, need, o.mass_before, s, d_mass, d_count, &pick, &found, &kept);
            have_slices = false;
        }
        if (o.by_count && p.p < 1.0) {      // top-p within the first k
            const double need = fmax(p.p * double(kept), 1.0);
            if (need > double(o.mass_before)) {       // it ends in the same bin
                if (o.mode == BIN) {
                    u64 got;
                    n = ranks_before(n, o.mass_before, need, &got);
                    least_key = list[n - 1];
                } else {
                    u64 got;
                    const u64 key = by_digits(l, a.vocab, p, o.last, false, need, o.mass_before, s, d_mass, d_count, &pick, &found, &got);
                    least_key = max(least_key, key);
                }
            } else {
                Plan e;
                find_bin<NT>(r, false, need, s, &shared, &e);
                u64 got;
                if (r.count[e.last] <= LIST) {
                    if (threadIdx.x == 0) listed = 0;
                    __syncthreads();
                    each<NT>(l, 0, a.vocab, [&](float x, int i) {
                        const double y = octaves(x, p);
                        if (weighs(y) && bin_of(y) == e.last) list[atomicAdd(&listed, 1u)] = rank_key(x, i);
                    });
                    __syncthreads();
                    n = int(listed);
                    int up = 2;
                    while (up < n) up <<= 1;
                    for (int i = n + int(threadIdx.x); i < up; i += NT) list[i] = 0;
                    sort_down(list, up);
                    n = ranks_before(n, e.mass_before, need, &got);
                    least_key = list[n - 1];
                } else {
                    least_key = by_digits(l, a.vocab, p, e.last, false, need, e.mass_before, s, d_mass, d_count, &pick, &found, &got);
                }
                have_slices = false;
            }
        }
    }
    auto weight_of = [&](float x, int i) -> u64 {
        const u64 w = weight(x, p);
        return w >= p.least && rank_key(x, i) >= least_key ? w : 0;
    };
    // the parts' weights: known but for the list's tokens, or summed here
    const int parts = a.slices * 4, part_len = (a.slice_len + 3) / 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto begin_of = [&](int i) { return min(min(a.vocab, (i / 4 + 1) * a.slice_len), i / 4 * a.slice_len + i % 4 * part_len); };
    auto end_of = [&](int i) { return min(min(a.vocab, (i / 4 + 1) * a.slice_len), i / 4 * a.slice_len + (i % 4 + 1) * part_len); };
    __syncthreads();
    if (have_slices) {
        for (int i = threadIdx.x; i < parts; i += NT) d_mass[i] = r.part_mass[i];
        __syncthreads();
        if (o.mode == BIN)
            for (int i = threadIdx.x; i < int(r.count[o.last]); i += NT) {
                const u64 k = list[i], w = weight(unorder(unsigned(k >> 32)), p);
                const int id = int(~unsigned(k)), in = id % a.slice_len;
                if (k >= least_key && w >= p.least) atomicAdd(&d_mass[id / a.slice_len * 4 + in / part_len], w);
            }
    } else {
        for (int i = wave; i < parts; i += NW) {
            u64 sum = 0;
            each<64>(l, begin_of(i), end_of(i), [&](float x, int j) { sum += weight_of(x, j); });
            sum = wave_sum(sum);
            if (lane == 0) d_mass[i] = sum;
        }
    }
    __syncthreads();
    // four parts a lane
    u64 own[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { own[i] = lane * 4 + i < parts ? d_mass[lane * 4 + i] : 0; mine += own[i]; }
    const u64 run = wave_scan(mine), total = last_lane(run);
    u64 target = place(total);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(run > target));
    target -= wave_sum(lane < at ? mine : 0);
    int part = at * 4;
    for (; part < at * 4 + 3 && target >= d_mass[part]; ++part) target -= d_mass[part];
    __syncthreads();
    const int id = first_past(l, weight_of, begin_of(part), end_of(part), target, s, &found);
    done(id, total);
}
}  // namespace

hipError_t launch_sample(const SampleArgs& x, void* ws, size_t ws_bytes, hipStream_t st) {
    const int at_once = int(std::min<size_t>(size_t(x.rows), ws_bytes / sizeof(Row)));
    if (at_once < 1) return hipErrorInvalidValue;
    for (int r0 = 0; r0 < x.rows; r0 += at_once) {
        const int n = std::min(at_once, x.rows - r0);
        // slices of 2048 logits or more, about 1024 workgroups
        int slices = std::min(SLICES, std::min((x.vocab + 2047) / 2048, (1024 + n - 1) / n));
        const int len = (x.vocab + slices - 1) / slices;
        slices = (x.vocab + len - 1) / len;
        const Args a = {x.logits + size_t(r0) * x.row_stride, x.row_stride, x.vocab, slices, len, x.temperature ? x.temperature + r0 : nullptr,
                        x.top_k ? x.top_k + r0 : nullptr, x.top_p ? x.top_p + r0 : nullptr, x.min_p ? x.min_p + r0 : nullptr, x.u + r0,
                        x.tokens + r0, x.logprobs ? x.logprobs + r0 : nullptr, (Row*)ws};
        hipLaunchKernelGGL(sample_max_kernel, dim3(unsigned(n * slices)), dim3(256), 0, st, a);
        hipLaunchKernelGGL(sample_bins_kernel, dim3(unsigned(n * slices)), dim3(256), 0, st, a);
        if (x.top_k || x.top_p) hipLaunchKernelGGL(sample_gather_kernel, dim3(unsigned(n * slices)), dim3(256), 0, st, a);
        hipLaunchKernelGGL(sample_pick_kernel, dim3(unsigned(n)), dim3(NT), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace cake
