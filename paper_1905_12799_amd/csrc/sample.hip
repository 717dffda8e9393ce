// A draw per row of logits with temperature, top-k, top-p and min-p (rls.h gives the rules).
//
// With d = (x - x_max) / temperature every rule but min-p is a cut in the order of descending d, equal ones by index.  -d is
// not negative, so its bits (the key) order like it does; key and index in one word are the entry's place, no two alike, and
// a cut is a place: what lies up to it is kept.  Weights are whole numbers, so their sums do not depend on who adds what.
//
// Reading the logits bounds it, 2 or 4 bytes for a maximum, an exponential and a sum.  What is done with a row goes by its length:
// - up to kThreadRow entries a thread takes a row, in registers, places counted against each other; up to kLaneRow 16 lanes do, two to four entries each;
// - up to kGroupRow a workgroup of 64 to 1024 threads takes a row, read once into registers, a thread 4 to 16 entries in a row of
//   them.  A cut is found by a histogram over d (counts and weights in LDS) and, in the bin it lies in, by counting the places
//   before each; where a bin holds more than fit the list in LDS, it is cut into bins of places, again and again.
// - longer rows are cut into chunks, a workgroup each; a launch for each of the passes.
// What it takes, of that the reading of the logits at the rate of a large copy: 524288 x 3 10 us (2), 524288 x 20 52 (8), 8 x 2000 with
// top-k and top-p 12, 2048 x 8000 44 (13), 64 x 128003 in bf16 with every rule 47 (3), 64 x 262144 with top-p 75 (13), 1 x 8388608 25 (7).
#include <algorithm>
#include <type_traits>
#include <utility>

#include "element_types.h"
#include "rls_internal.h"
#include "wave.h"

namespace rls {

namespace {

constexpr uint32_t kMaskedKey = 0x7f800000u;            // the key of what is never drawn

struct SampleArgs {
    const void *logits;
    int64_t rows, n, ld;
    const float *uniform, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *token;
    float *logprob;
};

// The settings of a row
struct RowRules {
    float inv;                                          // 1 / temperature
    int64_t k;                                          // entries of top-k (n: all)
    float p, least;                                     // of top-p (1: all), min-p (0: all; 1 at most, which is what the largest have)
    double u;
};
__device__ inline RowRules rules_of(const SampleArgs &a, int64_t row)
{
    // (every setting is read, from the numbers drawn where there is none, so that the reads are under way together)
    const float *const none = a.uniform;
    const float u = a.uniform[row], t = (a.temperature ? a.temperature : none)[row], p = (a.top_p ? a.top_p : none)[row],
                m = (a.min_p ? a.min_p : none)[row];
    const int32_t k = (a.top_k ? a.top_k : reinterpret_cast<const int32_t *>(none))[row];
    RowRules r;
    const bool greedy = a.temperature && !(t > 0.0f);
    r.k = greedy ? 1 : (a.top_k && k >= 1 && k < a.n ? (int64_t)k : a.n);
    r.inv = a.temperature && !greedy ? fminf(1.0f / t, 3.4028235e38f) : 1.0f;
    r.p = a.top_p && p < 1.0f ? p : 1.0f;
    r.least = a.min_p && m > 0.0f ? fminf(m, 1.0f) : 0.0f;
    r.u = u > 0.0f ? (double)u : 0.0;
    return r;
}

// (NaN counts as -infinity)
template <typename T>
__device__ inline float logit_of(T x)
{
    const float v = (float)x;
    return v == v ? v : -INFINITY;
}
// -d: 0 for the largest, infinite (or no number) for what is never drawn
__device__ inline float distance_from(float top, float x, float inv)
{
    if (top == INFINITY) return x == INFINITY ? 0.0f : INFINITY;
    return (top - x) * inv;
}
__device__ inline uint32_t key_of(float distance) { return distance < INFINITY ? __float_as_uint(distance) : kMaskedKey; }
__device__ inline float distance_of(uint32_t key) { return __uint_as_float(key); }

// exp(-distance) = 2^(-distance log2 e), the logarithm in two pieces: an exponential of the hardware and eight operations.  (Without what a
// general one does about results beyond the largest and below the smallest normal number: weights end at 2^-38, and beyond 100, at
// infinity and where there is no number this is exp(-100), which is no weight.  The steps are those of this target's expf, so that its weights are those of expf.)
__device__ inline float exp_of(float x)
{
    const float distance = fminf(x, 100.0f);
    constexpr float kHi = 0x1.715476p+0f, kLo = 0x1.4ae0bep-26f;
    const float whole = distance * -kHi, n = rintf(whole);
    const float rest = fmaf(distance, -kLo, fmaf(distance, -kHi, -whole));
    return ldexpf(__builtin_amdgcn_exp2f((whole - n) + rest), (int)n);
}

// Weight of an entry: its exponential in multiples of 2^-38 (adding 1.5 * 2^14 leaves the whole number in the low bits of a double).  Sums of
// many leave that offset in and take it off at the end, once per summand.
constexpr double kOffset = 1.5 * 16384.0;
__device__ inline uint64_t raw_weight(float e) { return (uint64_t)__double_as_longlong((double)e + kOffset); }
__device__ inline uint64_t offsets(uint64_t n) { return n * (uint64_t)__double_as_longlong(kOffset); }
__device__ inline uint64_t weight_of(float e) { return raw_weight(e) - offsets(1); }
__device__ inline uint64_t weight_of_key(uint32_t key) { return weight_of(exp_of(distance_of(key))); }
// whether an entry with so many entries, or so much weight, before it is inside top-k, or top-p (the first one always is)
__device__ inline bool begins_below(bool by_mass, uint64_t before, uint64_t k, double limit)
{
    return by_mass ? (before == 0) | ((double)before < limit) : before < k;
}
// Bins of a histogram: equal parts of the distances up to the widest, or up to 40 (beyond, exp(d) counts for nothing and only top-k
// can cut: with masks of the type's lowest value the bins keep their use); the last one takes the rest.
__device__ inline float bin_scale(float widest, int bins)
{
    const float width = fminf(widest, 40.0f);
    return width > 0.0f ? fminf((float)bins / width, 3e38f) : 0.0f;
}
__device__ inline int bin_of(uint32_t key, float scale, int bins) { return (int)fminf(distance_of(key) * scale, (float)(bins - 1)); }
__device__ inline float log_of(uint64_t total) { return logf((float)((double)total * 0x1p-38)); }

// Weight and count of the entries before one, up to 64 of them, as one number of 64 bits: the weights, whole numbers whose sum is 2^44 at
// most, and in the eight bits below them how many there are.  (Where an entry is not counted only its upper word is set to nothing: what
// is left is less than 2^-1022, which adds nothing to 1/256 and more.)
__device__ inline double counted_mass(uint64_t w) { return (double)w + 1.0 / 256.0; }
__device__ inline double mass_if(bool counted, uint64_t bits) { return __hiloint2double(counted ? (int)(bits >> 32) : 0, (int)bits); }
__device__ inline uint32_t count_of(double mass) { return (uint32_t)((mass - trunc(mass)) * 256.0); }

__device__ inline void no_draw(const SampleArgs &a, int64_t row)
{
    a.token[row] = -1;
    if (a.logprob) a.logprob[row] = -INFINITY;
}

// ---- short rows -----------------------------------------------------------------------------------

constexpr int kThreadRow = 16;

template <typename T, int V>
__global__ void __launch_bounds__(256) sample_short_kernel(SampleArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const int n = (int)a.n;
    float l[V];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        l[i] = logit_of(x[min(i, n - 1)]);
        if (i >= n) l[i] = -INFINITY;
        top = fmaxf(top, l[i]);
    }
    if (top == -INFINITY) { no_draw(a, row); return; }
    const RowRules r = rules_of(a, row);
    uint32_t key[V];
    float e[V];
    uint64_t w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        key[i] = key_of(distance_from(top, l[i], r.inv));
        e[i] = exp_of(distance_of(key[i]));
        w[i] = key[i] < kMaskedKey ? weight_of(e[i]) : 0;
    }
    if (r.k < n || r.p < 1.0f) {
        uint64_t mass[V], total = 0;
        double before[V];
        uint32_t in = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) mass[i] = (uint64_t)__double_as_longlong(counted_mass(w[i]));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            before[i] = 0.0;
#pragma unroll
            for (int j = 0; j < V; ++j) before[i] += j == i ? 0.0 : mass_if(key[j] < key[i] + (j < i ? 1u : 0u), mass[j]);
            const int rank = (int)count_of(before[i]);
            before[i] = trunc(before[i]);
            // (where an entry is inside top-k so is everything before it)
            in |= (rank < r.k ? 1u : 0u) << i;
            total += rank < r.k ? w[i] : 0;
        }
        const double limit = (double)r.p * (double)total;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            // (a selection, no branches: hipcc 7.2 loses the assignment of an element of an array in registers behind nested conditions)
            const bool out = ((in >> i & 1u) == 0) | ((r.p < 1.0f) & (before[i] > 0.0) & (before[i] >= limit));
            w[i] = out ? 0 : w[i];
        }
    }
    uint64_t total = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = (e[i] < r.least) & (key[i] != 0) ? 0 : w[i];
        total += w[i];
    }
    const double mark = r.u * (double)total;
    uint64_t run = 0;
    int token = -1;
    float d_token = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        run += w[i];
        const bool here = (token < 0) & (((double)run > mark) | (run == total));
        token = here ? i : token;
        d_token = here ? -distance_of(key[i]) : d_token;
    }
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = d_token - log_of(total);
}

// ---- rows of up to 64 entries ----------------------------------------------------------------------

constexpr int kLaneRow = 64;

// 16 lanes take a row, two to four entries each; for a cut every entry is counted against those of the 15 other lanes, which go round: 16 E^2
// pairs a lane, whose comparisons and additions are what bounds it.  524288 rows of 20, 40 and 64 entries without a cut 52, 63 and 72 us (reading
// the logits 8, 16 and 26), with top-k 91, 139 and 199, with top-p 133, 213 and 300; with four entries a lane for every length, 64-bit weights and
// ranks beside them top-k took 575 and top-p 625 at each.  (A wave per row: 524288 x 20 entries without a cut 330 us.)
template <typename T, int E>
__global__ void __launch_bounds__(256) sample_lanes_kernel(SampleArgs a)
{
    const int lane = threadIdx.x & 15, n = (int)a.n, first = lane * E;
    const int64_t at = (int64_t)blockIdx.x * (256 / 16) + (threadIdx.x >> 4), row = min(at, a.rows - 1);
    const RowRules r = rules_of(a, row);
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    float l[E], top = -INFINITY;
    if (first + E <= n) {
        T v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = x[first + j];
#pragma unroll
        for (int j = 0; j < E; ++j) l[j] = logit_of(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            l[j] = logit_of(x[min(first + j, n - 1)]);
            l[j] = first + j < n ? l[j] : -INFINITY;
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) top = fmaxf(top, l[j]);
    top = row_reduce(top, [](float u, float v) { return fmaxf(u, v); });
    uint32_t key[E];
    uint64_t w[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        key[j] = key_of(distance_from(top, l[j], r.inv));
        w[j] = key[j] < kMaskedKey ? weight_of_key(key[j]) : 0;
    }
    auto add = [](uint64_t u, uint64_t v) { return u + v; };
    const bool cut = (r.k < n) | (r.p < 1.0f);
    if (__any(cut)) {
        const bool by_mass = __any(r.p < 1.0f);
        // (what comes before an entry: by weight, both sums in one number)
        uint32_t rank[E] = {};
        double mass[E], before[E] = {};
#pragma unroll
        for (int j = 0; j < E; ++j) mass[j] = counted_mass(w[j]);
        auto against = [&](auto turn, auto weighed) {
            constexpr int s = decltype(turn)::value;
            constexpr bool kMass = decltype(weighed)::value;
            const bool earlier = lane >= s && s > 0;    // (row_ror:s brings the entries of lane - s, or of lane + 16 - s)
            uint32_t below[E];
#pragma unroll
            for (int j = 0; j < E; ++j) below[j] = key[j] + (earlier ? 1u : 0u);
#pragma unroll
            for (int o = 0; o < E; ++o) {
                const uint32_t key_o = s == 0 ? key[o] : lane_move<0x120 + (s ? s : 1), 0xf>(key[o], key[o]);
                const uint64_t bits = (uint64_t)__double_as_longlong(mass[o]);
                const uint64_t moved = !kMass || s == 0 ? bits : lane_move<0x120 + (s ? s : 1), 0xf>(bits, bits);
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const bool comes_first = key_o < (s == 0 && o < j ? key[j] + 1u : below[j]);
                    if constexpr (kMass) before[j] += mass_if(comes_first, moved);
                    else rank[j] += comes_first ? 1u : 0u;
                }
            }
        };
        auto all_turns = [&]<int... S>(std::integer_sequence<int, S...>, auto weighed) { (against(std::integral_constant<int, S>(), weighed), ...); };
        if (by_mass) {
            all_turns(std::make_integer_sequence<int, 16>(), std::true_type());
#pragma unroll
            for (int j = 0; j < E; ++j) {
                rank[j] = count_of(before[j]);
                before[j] = trunc(before[j]);
            }
        } else {
            all_turns(std::make_integer_sequence<int, 16>(), std::false_type());
        }
        uint64_t kept = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            w[j] = rank[j] < (uint32_t)r.k ? w[j] : 0;  // (where an entry is inside top-k so is everything before it)
            kept += w[j];
        }
        if (by_mass) {
            const double limit = (double)r.p * (double)row_reduce(kept, add);
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = (r.p < 1.0f) & (before[j] > 0.0) & (before[j] >= limit) ? 0 : w[j];
        }
    }
    uint64_t mine = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float e = exp_of(distance_of(key[j]));
        w[j] = (e < r.least) & (key[j] != 0) ? 0 : w[j];
        mine += w[j];
    }
    uint64_t run = row_scan(mine, (uint64_t)0, add);
    const uint64_t total = row_reduce(mine, add);
    const double mark = r.u * (double)total;
    auto beyond = [&](uint64_t v) { return ((double)v > mark) | (v == total); };
    run -= mine;
    int token = -1;
    uint32_t key_token = 0;
    const bool here = beyond(run + mine) & !beyond(run);
#pragma unroll
    for (int j = 0; j < E; ++j) {
        run += w[j];
        const bool now = (token < 0) & beyond(run);
        token = now ? first + j : token;
        key_token = now ? key[j] : key_token;
    }
    if (at >= a.rows) return;
    if (!(top > -INFINITY)) {
        if (lane == 0) no_draw(a, row);
    } else if (here) {
        a.token[row] = token;
        if (a.logprob) a.logprob[row] = -distance_of(key_token) - log_of(total);
    }
}

// ---- a workgroup's tools --------------------------------------------------------------------------

template <int NT>
struct Group {
    static constexpr int kWaves = NT / 64;
    static constexpr int kBins = NT == 64 ? 256 : 1024;
    // places that are counted against each other, by so many threads each (1000 by 1000 threads took 12 us, 256 by 1024 take one)
    static constexpr int kList = NT == 64 ? 128 : 256;
    static constexpr int kShare = NT > kList ? NT / kList : 1;
    static constexpr int kBinsOfThread = kBins / NT;

    struct Waves {
        uint64_t a[kWaves], b[kWaves];
    };
    struct Shared {
        uint64_t mass[kBins];
        uint32_t count[kBins];
        uint64_t place[kList], weight[kList], run[kList];
        Waves waves;
        uint64_t found_before;
        uint32_t found_bin, found_n, listed;
    };

    static __device__ inline void sync()
    {
        if constexpr (NT == 64) __builtin_amdgcn_wave_barrier();
        __syncthreads();
    }
    // reductions and scans over the workgroup; the results are the same in every thread
    template <typename F>
    static __device__ inline uint64_t reduce(Waves &waves, uint64_t x, F join)
    {
        x = wave_reduce(x, (uint64_t)0, join);
        if constexpr (NT > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) waves.a[threadIdx.x >> 6] = x;
            __syncthreads();
            x = waves.a[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) x = join(x, waves.a[w]);
        }
        return x;
    }
    static __device__ inline uint64_t sum(Shared &s, uint64_t x)
    {
        return reduce(s.waves, x, [](uint64_t a, uint64_t b) { return a + b; });
    }
    static __device__ inline uint64_t most(Shared &s, uint64_t x)
    {
        return reduce(s.waves, x, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    }
    // the largest of one value and the smallest of another
    static __device__ inline void range(Shared &s, float &top, float &low)
    {
        top = wave_max(top);
        low = wave_min(low);
        if constexpr (NT > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s.waves.a[threadIdx.x >> 6] = (uint64_t)__float_as_uint(top) << 32 | __float_as_uint(low);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                top = fmaxf(top, __uint_as_float((uint32_t)(s.waves.a[w] >> 32)));
                low = fminf(low, __uint_as_float((uint32_t)s.waves.a[w]));
            }
        }
    }
    // what the threads before this one have (and the sum of all)
    static __device__ inline uint64_t scan(Waves &waves, uint64_t x, uint64_t *total)
    {
        const uint64_t run = wave_scan(x, (uint64_t)0, [](uint64_t a, uint64_t b) { return a + b; });
        if constexpr (NT == 64) {
            *total = last_lane(run);
            return run - x;
        } else {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
            __syncthreads();
            if (lane == 63) waves.b[wave] = run;
            __syncthreads();
            uint64_t before = 0, all = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint64_t v = waves.b[w];
                before += w < wave ? v : 0;
                all += v;
            }
            *total = all;
            return before + run - x;
        }
    }

    static __device__ inline void clear(Shared &s)
    {
        sync();
#pragma unroll
        for (int b = 0; b < kBinsOfThread; ++b) {
            s.count[threadIdx.x * kBinsOfThread + b] = 0;
            s.mass[threadIdx.x * kBinsOfThread + b] = 0;
        }
        sync();
    }
    // The last bin whose entries begin below: fewer than k entries before it, or less weight than `limit`, of which `base` come before all
    // bins.  Leaves the bin, its entries, and entries or weight before it in s.
    static __device__ inline void find_bin(Shared &s, bool by_mass, uint64_t k, double limit, uint64_t base)
    {
        if (threadIdx.x == 0) s.found_bin = 0;
        sync();
        uint64_t mine = 0, all;
#pragma unroll
        for (int b = 0; b < kBinsOfThread; ++b) {
            const int i = threadIdx.x * kBinsOfThread + b;
            mine += by_mass ? s.mass[i] : s.count[i];
        }
        const uint64_t before = base + scan(s.waves, mine, &all);
        int last = -1;
        uint64_t run = before, last_run = 0;
#pragma unroll
        for (int b = 0; b < kBinsOfThread; ++b) {
            const int i = threadIdx.x * kBinsOfThread + b;
            const uint32_t n = s.count[i];
            const bool below = (n > 0) & begins_below(by_mass, run, k, limit);
            last = below ? i : last;
            last_run = below ? run : last_run;
            run += by_mass ? s.mass[i] : n;
        }
        if (last >= 0) atomicMax(&s.found_bin, (uint32_t)last);
        sync();
        if (last >= 0 && s.found_bin == (uint32_t)last) {
            s.found_n = s.count[last];
            s.found_before = last_run;
        }
        sync();
    }
    // entries or weight of the list's places from..to that come before `at`
    static __device__ inline uint64_t smaller(const Shared &s, uint64_t at, uint32_t from, uint32_t to, bool by_mass)
    {
        uint64_t run = 0;
#pragma unroll 8
        for (uint32_t o = from; o < to; ++o) {
            const uint64_t add = by_mass ? s.weight[o] : 1;
            run += s.place[o] < at ? add : 0;
        }
        return run;
    }
    // Among the n entries that `visit` hands to a function of place and key, the last place that begins below (see find_bin).  Where they fit the
    // list they are counted against each other; more are cut into bins of places first, again and again.
    template <typename Visit>
    static __device__ inline uint64_t last_below(Shared &s, Visit visit, uint64_t n, bool by_mass, uint64_t k, double limit, uint64_t before)
    {
        uint64_t lo = 0, hi = ~0ull;
        if (n > kList) {
            uint64_t first = ~0ull, last = 0;
            visit([&](uint64_t at, uint32_t) {
                first = first < at ? first : at;
                last = last > at ? last : at;
            });
            lo = ~most(s, ~first);
            hi = most(s, last);
        }
        while (n > kList && lo < hi) {
            const uint64_t spread = hi - lo;
            const int bits = 64 - __clzll((long long)spread);
            int shift = bits - (kBins == 256 ? 8 : 10);
            shift = shift > 0 ? shift : 0;
            clear(s);
            visit([&](uint64_t at, uint32_t key) {
                if (at < lo || at > hi) return;
                const int b = (int)((at - lo) >> shift);
                atomicAdd(&s.count[b], 1u);
                if (by_mass) atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[b]), (unsigned long long)weight_of_key(key));
            });
            find_bin(s, by_mass, k, limit, before);
            lo += (uint64_t)s.found_bin << shift;
            const uint64_t end = lo + ((1ull << shift) - 1);
            hi = end < hi ? end : hi;
            n = s.found_n;
            before = s.found_before;
            sync();
        }
        if (lo == hi) return lo;
        if (threadIdx.x == 0) s.listed = 0;
        sync();
        visit([&](uint64_t at, uint32_t key) {
            if (at < lo || at > hi) return;
            const uint32_t i = atomicAdd(&s.listed, 1u);
            s.place[i] = at;
            s.weight[i] = weight_of_key(key);
        });
        sync();
        const uint32_t listed = s.listed;
        uint64_t cut = 0;
        if constexpr (kShare == 1) {
            for (uint32_t i = threadIdx.x; i < listed; i += NT) {
                const uint64_t at = s.place[i], run = before + smaller(s, at, 0, listed, by_mass);
                if (begins_below(by_mass, run, k, limit)) cut = cut > at ? cut : at;
            }
        } else {
            const uint32_t i = threadIdx.x % kList, share = threadIdx.x / kList, part = (listed + kShare - 1) / kShare;
            if (share == 0) s.run[i] = before;
            __syncthreads();
            const uint64_t at = s.place[i];
            if (i < listed)
                atomicAdd(reinterpret_cast<unsigned long long *>(&s.run[i]), (unsigned long long)smaller(s, at, share * part, min(listed, share * part + part), by_mass));
            __syncthreads();
            if (share == 0 && i < listed && begins_below(by_mass, s.run[i], k, limit)) cut = at;
        }
        return most(s, cut);
    }

    // Entries in registers: their keys and the index of the first one (the others follow).  Exponentials and weights are computed
    // where they are needed, four at a time, and forgotten: all at once they do not fit the 128 registers of a thread of 1024.
    static __device__ inline void pace(int j)
    {
        if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    template <int E>
    struct Entries {
        uint32_t key[E];
        uint32_t first;
        __device__ inline uint64_t place(int j) const { return (uint64_t)key[j] << 32 | (first + (uint32_t)j); }
        __device__ inline bool there(int j) const { return key[j] < kMaskedKey; }
        // (compared as two halves: 64-bit places of all entries would be register pairs beside the keys)
        __device__ inline bool upto(int j, uint64_t cut) const
        {
            const uint32_t k = (uint32_t)(cut >> 32);
            return key[j] < k || (key[j] == k && first + (uint32_t)j <= (uint32_t)cut);
        }
        __device__ inline void forget()
        {
#pragma unroll
            for (int j = 0; j < E; ++j) asm volatile("" : "+v"(key[j]));
        }
    };

    // The cut of top-k and top-p over the entries, the furthest `widest` away from the largest.
    template <int E>
    static __device__ inline uint64_t cut_of(Shared &s, Entries<E> &x, float widest, uint64_t k, bool use_k, float p, bool use_p)
    {
        const float scale = bin_scale(widest, kBins);
        clear(s);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (x.there(j)) {
                const int b = bin_of(x.key[j], scale, kBins);
                atomicAdd(&s.count[b], 1u);
                if (use_p) atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[b]), (unsigned long long)weight_of_key(x.key[j]));
            }
            pace(j);
        }
        uint64_t cut = ~0ull;
        // (the list's places overwrite no bin, and a second cut begins from the same bins unless the first one had to cut its bin up)
        auto in_bin = [&](int bin, bool by_mass, double limit, uint64_t n, uint64_t before) {
            return last_below(s, [&](auto what) {
                x.forget();
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (x.there(j) && bin_of(x.key[j], scale, kBins) == bin && x.upto(j, cut)) what(x.place(j), x.key[j]);
                    pace(j);
                }
            }, n, by_mass, k, limit, before);
        };
        if (use_k) {
            find_bin(s, false, k, 0.0, 0);
            const bool crowded = s.found_n > kList;
            cut = in_bin((int)s.found_bin, false, 0.0, s.found_n, s.found_before);
            if (use_p && crowded) {
                clear(s);
                x.forget();
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (x.there(j)) {
                        const int b = bin_of(x.key[j], scale, kBins);
                        atomicAdd(&s.count[b], 1u);
                        atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[b]), (unsigned long long)weight_of_key(x.key[j]));
                    }
                    pace(j);
                }
            }
        }
        if (use_p) {
            uint64_t kept = 0;
            x.forget();
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (x.there(j) && x.upto(j, cut)) kept += weight_of_key(x.key[j]);
                pace(j);
            }
            const double limit = (double)p * (double)sum(s, kept);
            // (a bin that begins below the limit begins no later than the cut's)
            find_bin(s, true, 0, limit, 0);
            cut = in_bin((int)s.found_bin, true, limit, s.found_n, s.found_before);
        }
        return cut;
    }
};

// ---- rows in registers ----------------------------------------------------------------------------

template <typename T, int NT, int E>
__global__ void __launch_bounds__(NT) sample_row_kernel(SampleArgs a)
{
    using Grp = Group<NT>;
    __shared__ typename Grp::Shared s;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Grp::sync();
        const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
        const int n = (int)a.n, first = (int)threadIdx.x * E;
        constexpr int N = 16 / sizeof(T) < E ? 16 / sizeof(T) : E;      // elements of a load
        float l[E];
#pragma unroll
        for (int q = 0; q < E; q += N) {
            if (first + q + N <= n) {
                T v[N];
                __builtin_memcpy(v, x + first + q, sizeof(v));
#pragma unroll
                for (int j = 0; j < N; ++j) l[q + j] = logit_of(v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) l[q + j] = first + q + j < n ? logit_of(x[first + q + j]) : -INFINITY;
            }
        }
        const RowRules r = rules_of(a, row);
        float top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            top = fmaxf(top, l[j]);
            low = fminf(low, l[j] > -INFINITY ? l[j] : INFINITY);
        }
        Grp::range(s, top, low);
        if (top == -INFINITY) {
            if (threadIdx.x == 0) no_draw(a, row);
            continue;
        }
        typename Grp::template Entries<E> entry;
        entry.first = (uint32_t)first;
#pragma unroll
        for (int j = 0; j < E; ++j) entry.key[j] = key_of(distance_from(top, l[j], r.inv));
        uint64_t cut = ~0ull;
        if (r.k < n || r.p < 1.0f) cut = Grp::cut_of(s, entry, distance_from(top, low, r.inv), (uint64_t)r.k, r.k < n, r.p, r.p < 1.0f);
        auto weight = [&](int j) -> uint64_t {
            if (!entry.there(j) || !entry.upto(j, cut)) return 0;
            const float e = exp_of(distance_of(entry.key[j]));
            return e < r.least && entry.key[j] != 0 ? 0 : weight_of(e);
        };
        uint64_t mine = 0, total;
        entry.forget();
#pragma unroll
        for (int j = 0; j < E; ++j) {
            mine += weight(j);
            Grp::pace(j);
        }
        uint64_t run = Grp::scan(s.waves, mine, &total);
        const double mark = r.u * (double)total;
        auto beyond = [&](uint64_t v) { return (double)v > mark || v == total; };
        if (beyond(run + mine) && !beyond(run)) {
            bool open = true;
            entry.forget();
#pragma unroll
            for (int j = 0; j < E; ++j) {
                run += weight(j);
                if (open && beyond(run)) {
                    open = false;
                    a.token[row] = (int32_t)(first + j);
                    if (a.logprob) a.logprob[row] = -distance_of(entry.key[j]) - log_of(total);
                }
                Grp::pace(j);
            }
        }
    }
}

constexpr int64_t kGroupRow = 16384;
// (8 x 2000 with top-k and top-p: 256 threads of 16 entries 21 us where 512 of 4 take 12; 2048 x 8000: 1024 of 16 77 us, 512 of 16 45.  Rows from
// 16385 on: 512 x 32768 103 us by workgroups of a row, 42 in chunks; 1024 x 16384 53 and 66.)
constexpr int64_t kFewRows = 512;
constexpr int64_t kMostGroups = 1 << 20;           // (of a launch, which ends at 2^32 threads)

template <typename T>
hipError_t launch_group_rows(const SampleArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows < kMostGroups ? a.rows : kMostGroups));
    // a few rows are as long as what a thread does in turn: four entries each; many rows are work, of which a larger workgroup has more in its
    // scans and barriers
    const bool few = a.rows <= kFewRows;
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a); };
    if (a.n <= 256) launch(sample_row_kernel<T, 64, 4>, 64);
    else if (a.n <= 1024) few ? launch(sample_row_kernel<T, 256, 4>, 256) : a.n <= 512 ? launch(sample_row_kernel<T, 64, 8>, 64) : launch(sample_row_kernel<T, 64, 16>, 64);
    else if (a.n <= 2048) few ? launch(sample_row_kernel<T, 512, 4>, 512) : launch(sample_row_kernel<T, 128, 16>, 128);
    else if (a.n <= 4096) few ? launch(sample_row_kernel<T, 1024, 4>, 1024) : launch(sample_row_kernel<T, 256, 16>, 256);
    else if (a.n <= 8192) few ? launch(sample_row_kernel<T, 1024, 8>, 1024) : launch(sample_row_kernel<T, 512, 16>, 512);
    else launch(sample_row_kernel<T, 1024, 16>, 1024);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_short_rows(const SampleArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.rows + 255) / 256));
    if (a.n <= 4) hipLaunchKernelGGL((sample_short_kernel<T, 4>), grid, dim3(256), 0, s, a);
    else if (a.n <= 8) hipLaunchKernelGGL((sample_short_kernel<T, 8>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sample_short_kernel<T, kThreadRow>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// ---- long rows ------------------------------------------------------------------------------------

// Rows are cut into chunks, a workgroup each, and a batch of rows goes through launches: the maxima; where rows have top-k or top-p a
// histogram (of entries for top-k, of weights for top-p), and the bins that a row's cuts lie in; the weights of what lies before these bins, segment
// by segment, and the entries in them as a list; the cuts from the list, its share of the weights and the draw, a workgroup per row.
// What a launch needs of the row's other chunks it finds in the workspace.
constexpr int kLongThreads = 512;
constexpr int kLongWaves = kLongThreads / 64;
constexpr int kLongBins = 2048;
constexpr int64_t kLongList = 16384;                    // entries of a row's list, or a 64th of the row where that is more: ordinary logits have a 500th in a bin
inline int64_t list_of(int64_t n) { return std::max(kLongList, n / 64); }
constexpr int64_t kListedK = 4096;                      // top-k of so many at most: all it keeps goes through the list, weights and top-p with it
constexpr uint32_t kLdsList = 2048;                     // entries of it that the draw holds in LDS
constexpr int kLongStage = 1024;                        // places a workgroup collects before it goes to the row's list one by one
constexpr int64_t kLongRows = 256;                      // of a batch
constexpr int kMostPieces = 512;                        // chunks of a row
constexpr int kMostSegments = kMostPieces * kLongWaves; // a segment is a wave's part of a chunk
constexpr int kMostChunk = 65536;
constexpr int kLoad = 8;                                // entries a thread takes in a row

struct Piece {
    float top, low;                                     // the largest, and the smallest that is not masked
    uint32_t at;                                        // where the largest is first
};
struct RowBins {                                        // where a row's cuts lie
    int32_t k_bin, p_first, p_last;                     // top-k's bin; top-p's is one of these, which depends on what top-k keeps of its own
    float near, far, k_near, k_far;                     // distances: kept in any case before `near`; the bins' entries are from `near`, and `k_near`, on
    uint32_t k_count, k_before;
    uint64_t k_mass_before, p_mass_before;              // weight before k_bin, p_first
    uint64_t mass;                                      // of the row
    float scale;
};
struct InBins {                                         // of a segment: the entries in the bins of the row's cuts, the nearest and the furthest of them
    uint32_t n;
    float least, most;
};
struct LongArgs {
    SampleArgs a;
    int64_t row0, chunk;
    int32_t rows, pieces, list_size;
    Piece *piece;                                       // [rows][pieces]
    uint64_t *weight;                                   // [rows][pieces][kLongWaves]
    uint64_t *mass;                                     // [rows][kLongBins]
    uint32_t *count, *listed;                           // [rows][kLongBins], [rows]
    InBins *in_bins;                                    // [rows][pieces][kLongWaves]
    uint64_t *list;                                     // [rows][list_size]
    RowBins *bins;                                      // [rows]
};

// The entries of a span, kLoad at a time by each of `n` threads, with two loads of each under way; a thread's indices ascend.  (NaN comes as it is: no
// comparison takes it for a largest or smallest one, and its distance is none.)
template <typename T, typename F>
__device__ inline void visit_span(const T *x, int64_t begin, int64_t end, int thread, int n, F what)
{
    constexpr int U = 2 * 16 / (kLoad * (int)sizeof(T)) > 1 ? 4 : 2;
    const int64_t step = (int64_t)n * kLoad;
    int64_t i = begin + (int64_t)thread * kLoad;
    for (; i + (U - 1) * step + kLoad <= end; i += U * step) {
        T v[U][kLoad];
#pragma unroll
        for (int u = 0; u < U; ++u) __builtin_memcpy(v[u], x + i + u * step, sizeof(v[u]));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kLoad; ++j) what((float)v[u][j], i + u * step + j);
    }
    for (; i < end; i += step) {
        if (i + kLoad <= end) {
            T v[kLoad];
            __builtin_memcpy(v, x + i, sizeof(v));
#pragma unroll
            for (int j = 0; j < kLoad; ++j) what((float)v[j], i + j);
        } else {
            for (int64_t j = i; j < end; ++j) what((float)x[j], j);
        }
    }
}

__device__ inline Piece joined(const Piece &a, const Piece &b)
{
    return Piece{fmaxf(a.top, b.top), fminf(a.low, b.low), a.top > b.top ? a.at : (b.top > a.top ? b.at : min(a.at, b.at))};
}
__device__ inline Piece of_wave(const Piece &p)
{
    const float top = wave_max(p.top);
    const uint32_t at = wave_reduce(p.top == top ? p.at : ~0u, ~0u, [](uint32_t a, uint32_t b) { return min(a, b); });
    return Piece{top, wave_min(p.low), at};
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_top_kernel(LongArgs q)
{
    __shared__ Piece lds[kLongWaves];
    const int piece = blockIdx.x, r = blockIdx.y;
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    Piece p{-INFINITY, INFINITY, ~0u};
    visit_span(x, begin, end, threadIdx.x, kLongThreads, [&](float v, int64_t i) {
        p.at = v > p.top ? (uint32_t)i : p.at;
        p.top = fmaxf(p.top, v);
        p.low = fminf(p.low, v > -INFINITY ? v : INFINITY);
    });
    p = of_wave(p);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = p;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kLongWaves; ++w) p = joined(p, lds[w]);
        q.piece[(int64_t)r * q.pieces + piece] = p;
        if (piece == 0) q.listed[r] = 0;
    }
    // the row's histogram is cleared by its workgroups together
    if (q.a.top_k || q.a.top_p)
        for (int b = piece * kLongThreads + threadIdx.x; b < kLongBins; b += q.pieces * kLongThreads) {
            q.count[(int64_t)r * kLongBins + b] = 0;
            q.mass[(int64_t)r * kLongBins + b] = 0;
        }
}

// The whole row's largest entry, the first place it is at, and the smallest that is not masked: every wave for itself
__device__ inline Piece row_top(const LongArgs &q, int r)
{
    constexpr int U = kMostPieces / 64;                 // (all reads under way together)
    const Piece *const pieces = q.piece + (int64_t)r * q.pieces;
    const int lane = threadIdx.x & 63;
    Piece v[U], p{-INFINITY, INFINITY, ~0u};
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (64 * u < q.pieces) v[u] = pieces[min(64 * u + lane, q.pieces - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (64 * u < q.pieces) p = joined(p, v[u]);     // (one that is read twice changes nothing)
    return of_wave(p);
}

// whether all that top-k keeps goes through the list: its histogram needs no weights then
__device__ inline bool k_by_list(const LongArgs &q, const RowRules &r) { return r.k < q.a.n && r.k <= kListedK; }
// Whether a row's one entry is its largest, which is known from the maxima.  (Not where temperature brings other entries to a distance of 0: the
// one below the largest is at least 2^-25 of it, or the smallest number, away.)
__device__ inline bool is_top(const RowRules &r, float top) { return (r.k == 1) & (fmaxf(fabsf(top) * 0x1p-25f, 0x1p-149f) * r.inv > 0.0f); }
// whether a row's cut has to be looked for
__device__ inline bool cuts(const LongArgs &q, const RowRules &r, float top)
{
    return top > -INFINITY && !is_top(r, top) && (r.k < q.a.n || r.p < 1.0f);
}

// `what` with a function from logits to distances: where nothing is infinite it has no case for that
template <typename F>
__device__ inline void with_distances(float top, float inv, F what)
{
    if (top < INFINITY) what([=](float v) { return (top - v) * inv; });
    else what([=](float v) { return distance_from(top, v, inv); });
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_histogram_kernel(LongArgs q)
{
    __shared__ uint64_t mass[kLongBins];
    __shared__ uint32_t count[kLongBins];
    const int piece = blockIdx.x, r = blockIdx.y;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const Piece p = row_top(q, r);
    if (!cuts(q, rules, p.top)) return;
    const float scale = bin_scale(distance_from(p.top, p.low, rules.inv), kLongBins);
    for (int b = threadIdx.x; b < kLongBins; b += kLongThreads) { count[b] = 0; mass[b] = 0; }
    __syncthreads();
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    const bool use_k = rules.k < q.a.n, use_p = rules.p < 1.0f && !k_by_list(q, rules);
    with_distances(p.top, rules.inv, [&](auto distance) {
        visit_span(x, begin, end, threadIdx.x, kLongThreads, [&](float v, int64_t) {
            const float d = distance(v);
            if (!(d < INFINITY)) return;
            const int b = (int)fminf(d * scale, (float)(kLongBins - 1));
            if (use_k) atomicAdd(&count[b], 1u);
            if (use_p) atomicAdd(reinterpret_cast<unsigned long long *>(&mass[b]), (unsigned long long)weight_of(exp_of(d)));
        });
    });
    __syncthreads();
    uint32_t *const row_count = q.count + (int64_t)r * kLongBins;
    uint64_t *const row_mass = q.mass + (int64_t)r * kLongBins;
    for (int b = threadIdx.x; b < kLongBins; b += kLongThreads) {
        if (count[b]) atomicAdd(&row_count[b], count[b]);
        if (mass[b]) atomicAdd(reinterpret_cast<unsigned long long *>(&row_mass[b]), (unsigned long long)mass[b]);
    }
}

// The bins that a row's cuts lie in.  (Found by the last workgroup of the row to finish its histogram this took 100 us more: its fence
// writes the second-level cache back.)
__global__ void __launch_bounds__(kLongThreads) long_bins_kernel(LongArgs q)
{
    using Grp = Group<kLongThreads>;
    __shared__ typename Grp::Waves waves;
    __shared__ uint64_t around[2];
    __shared__ int32_t bin_k, bin_first, bin_last;
    const int r = blockIdx.x;
    const uint32_t *const row_count = q.count + (int64_t)r * kLongBins;
    const uint64_t *const row_mass = q.mass + (int64_t)r * kLongBins;
    constexpr int B = kLongBins / kLongThreads;
    uint32_t c_of[B];
    uint64_t m_of[B], n = 0, w = 0, all_n, all_w;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        c_of[b] = row_count[threadIdx.x * B + b];
        m_of[b] = row_mass[threadIdx.x * B + b];
        n += c_of[b];
        w += m_of[b];
    }
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const Piece p = row_top(q, r);
    if (!cuts(q, rules, p.top)) return;
    const bool use_k = rules.k < q.a.n, by_list = k_by_list(q, rules), use_p = rules.p < 1.0f && !by_list;
    const float scale = bin_scale(distance_from(p.top, p.low, rules.inv), kLongBins);
    const uint64_t n_before = Grp::scan(waves, n, &all_n), w_before = Grp::scan(waves, w, &all_w);
    if (threadIdx.x == 0) bin_k = bin_first = bin_last = -1;
    __syncthreads();
    // every bin with entries and weight in it and before it, by the thread that has it
    auto bins = [&](auto what) {
        uint64_t c = n_before, m = w_before;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            what((int)threadIdx.x * B + b, c_of[b], m_of[b], c, m);
            c += c_of[b];
            m += m_of[b];
        }
    };
    // the last bin that begins below
    auto last_bin = [&](int32_t *found, auto below) {
        int mine = -1;
        bins([&](int b, uint32_t c, uint64_t m, uint64_t c0, uint64_t m0) { mine = below(c, m, c0, m0) ? b : mine; });
        if (mine >= 0) atomicMax(found, mine);
        __syncthreads();
    };
    RowBins *const out = &q.bins[r];
    uint64_t least = all_w, most = all_w;               // weight that top-k keeps, at least and at most
    if (use_k) {
        last_bin(&bin_k, [&](uint32_t c, uint64_t, uint64_t c0, uint64_t) { return (c > 0) & (c0 < (uint64_t)rules.k); });
        bins([&](int b, uint32_t c, uint64_t m, uint64_t c0, uint64_t m0) {
            if (b != bin_k) return;
            around[0] = m0;
            around[1] = m0 + m;
            out->k_count = c;
            out->k_before = (uint32_t)c0;
            out->k_mass_before = m0;
        });
        __syncthreads();
        least = around[0];
        most = around[1];
    }
    if (use_p) {
        // (entries without weight are none that a nucleus ends with)
        const double limit_least = (double)rules.p * (double)least, limit_most = (double)rules.p * (double)most;
        last_bin(&bin_first, [&](uint32_t, uint64_t m, uint64_t, uint64_t m0) { return (m > 0) & begins_below(true, m0, 0, limit_least); });
        last_bin(&bin_last, [&](uint32_t, uint64_t m, uint64_t, uint64_t m0) { return (m > 0) & begins_below(true, m0, 0, limit_most); });
        bins([&](int b, uint32_t, uint64_t, uint64_t, uint64_t m0) {
            if (b == bin_first) out->p_mass_before = m0;
        });
    }
    // the least distance that falls into a bin, for the ends of the bins: next to the bin's number over the scale
    if (threadIdx.x < 4) {
        const int near = use_p ? bin_first : bin_k, far = use_p ? bin_last : bin_k;
        const int bin = threadIdx.x == 0 ? near : (threadIdx.x == 1 ? far + 1 : (threadIdx.x == 2 ? bin_k : bin_k + 1));
        uint32_t lo = 0;
        if (bin >= kLongBins) lo = kMaskedKey;
        else if (bin > 0) {
            lo = min(__float_as_uint((float)bin / scale), kMaskedKey - 1);
            while (lo > 0 && bin_of(lo - 1, scale, kLongBins) >= bin) --lo;
            while (lo < kMaskedKey && bin_of(lo, scale, kLongBins) < bin) ++lo;
        }
        (&out->near)[threadIdx.x] = by_list && threadIdx.x == 0 ? 0.0f : distance_of(lo);
    }
    if (threadIdx.x == 0) {
        out->k_bin = bin_k;
        out->p_first = bin_first;
        out->p_last = bin_last;
        out->mass = all_w;
        out->scale = scale;
    }
}

// what an entry adds to the draw, its place aside
__device__ inline uint64_t kept_weight(float distance, float least)
{
    const float e = exp_of(distance);
    return (e < least) & (distance != 0.0f) ? 0 : weight_of(e);
}

// The weights of a chunk's segments, as far as they lie before the bins of the row's cuts, and the entries in these bins.
template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_weight_kernel(LongArgs q)
{
    __shared__ uint64_t stage[kLongStage];
    __shared__ uint32_t staged, base;
    const int piece = blockIdx.x, r = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const float top = row_top(q, r).top;
    if (!(top > -INFINITY) || is_top(rules, top)) return;
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t segment = q.chunk / kLongWaves;
    const int64_t begin = min(q.a.n, piece * q.chunk + wave * segment), end = min(q.a.n, begin + segment);
    uint64_t w = 0;
    if (!cuts(q, rules, top)) {
        with_distances(top, rules.inv, [&](auto distance) {
            if (rules.least > 0.0f) {
                visit_span(x, begin, end, lane, 64, [&](float v, int64_t) { w += kept_weight(distance(v), rules.least); });
            } else {
                visit_span(x, begin, end, lane, 64, [&](float v, int64_t) { w += raw_weight(exp_of(distance(v))); });
            }
        });
        w = wave_sum(w) - (rules.least > 0.0f ? 0 : offsets((uint64_t)(end - begin)));
    } else {
        if (threadIdx.x == 0) staged = 0;
        __syncthreads();
        const float near = q.bins[r].near, far = q.bins[r].far, k_near = q.bins[r].k_near, k_far = q.bins[r].k_far;
        uint32_t in_bins = 0;
        float least = INFINITY, most = 0.0f;
        bool full = false;                              // the list (then nobody needs to know by how much)
        with_distances(top, rules.inv, [&](auto distance) {
            visit_span(x, begin, end, lane, 64, [&](float v, int64_t i) {
                const float d = distance(v);
                if (d < near) w += kept_weight(d, rules.least);
                else if ((d < far) | ((d >= k_near) & (d < k_far))) {
                    const uint64_t place = (uint64_t)__float_as_uint(d) << 32 | (uint32_t)i;
                    ++in_bins;
                    least = fminf(least, d);
                    most = fmaxf(most, d);
                    const uint32_t at = atomicAdd(&staged, 1u);
                    if (at < kLongStage) stage[at] = place;
                    else if (!full) {
                        const uint32_t to = atomicAdd(&q.listed[r], 1u);
                        full = to >= (uint32_t)q.list_size;
                        if (to < (uint32_t)q.list_size) q.list[(int64_t)r * q.list_size + to] = place;
                    }
                }
            });
        });
        in_bins = wave_reduce(in_bins, 0u, [](uint32_t a, uint32_t b) { return a + b; });
        least = wave_min(least);
        most = wave_max(most);
        if (lane == 0) q.in_bins[((int64_t)r * q.pieces + piece) * kLongWaves + wave] = InBins{in_bins, least, most};
        __syncthreads();
        const uint32_t own = staged < kLongStage ? staged : kLongStage;
        if (own > 0) {                                  // (the same in every thread)
            if (threadIdx.x == 0) base = atomicAdd(&q.listed[r], own);
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < own; i += kLongThreads)
                if (base + i < (uint32_t)q.list_size) q.list[(int64_t)r * q.list_size + base + i] = stage[i];
        }
        w = wave_sum(w);
    }
    if (lane == 0) q.weight[((int64_t)r * q.pieces + piece) * kLongWaves + wave] = w;
}

// The cuts, from the list.  Where a row's bins hold more entries than the list and these are all equal, so many of them are kept, counted segment by
// segment; where they are not (several values that lie close together, thousands of times each), a workgroup goes through the row, some five
// times, 3 ms each for 8 million entries.  Then the draw.
template <typename T>
__global__ void __launch_bounds__(1024) long_draw_kernel(LongArgs q)
{
    using Grp = Group<1024>;
    __shared__ typename Grp::Shared s;
    __shared__ uint64_t weight[kMostSegments], held[kLdsList];
    __shared__ int found;
    __shared__ uint64_t found_before;
    const int r = blockIdx.x;
    const int64_t row = q.row0 + r;
    if (threadIdx.x == 0) { found = 0; found_before = 0; }      // (a place inside the row in any case)
    const RowRules rules = rules_of(q.a, row);
    const Piece p = row_top(q, r);
    if (!(p.top > -INFINITY) || is_top(rules, p.top)) {
        if (threadIdx.x == 0) {
            if (p.top > -INFINITY) {
                q.a.token[row] = (int32_t)p.at;
                if (q.a.logprob) q.a.logprob[row] = 0.0f;
            } else no_draw(q.a, row);
        }
        return;
    }
    const T *const x = static_cast<const T *>(q.a.logits) + row * q.a.ld;
    const int64_t segment = q.chunk / kLongWaves;
    const int segments = q.pieces * kLongWaves;
    {
        constexpr int U = kMostSegments / 1024;
        uint64_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (1024 * u < segments) v[u] = q.weight[(int64_t)r * segments + min(1024 * u + (int)threadIdx.x, segments - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (1024 * u + (int)threadIdx.x < segments) weight[1024 * u + threadIdx.x] = v[u];
    }
    // a thread's part of a segment, in the order of the entries
    constexpr int S = kMostSegments / 1024, E = kMostChunk / kLongWaves / 1024;
    const int64_t part = (segment + 1023) / 1024;
    auto keys_of = [&](int which, uint32_t (&key)[E]) {
        const int64_t begin = which * segment, end = min(q.a.n, begin + segment), from = min(end, begin + part * threadIdx.x), to = min(end, from + part);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float v = logit_of(x[min(from + j, q.a.n - 1)]);
            key[j] = from + j < to ? key_of(distance_from(p.top, v, rules.inv)) : kMaskedKey;
        }
        return from;
    };
    uint64_t cut = ~0ull;
    const uint32_t listed = q.listed[r];
    const bool cut_it = cuts(q, rules, p.top);
    bool equal = false;
    uint32_t held_by[S], tied = 0;
    uint64_t mine = 0;
    if (cut_it && listed > (uint32_t)q.list_size) {
        float least = INFINITY, most = 0.0f;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int at = (int)threadIdx.x * S + i;
            const InBins in = at < segments ? q.in_bins[(int64_t)r * segments + at] : InBins{0, INFINITY, 0.0f};
            held_by[i] = in.n;
            mine += in.n;
            least = fminf(least, in.least);
            most = fmaxf(most, in.most);
        }
        Grp::range(s, most, least);
        equal = least == most;
        tied = __float_as_uint(most);
    }
    if (equal) {
        const RowBins bins = q.bins[r];
        __syncthreads();
        uint64_t all;
        uint64_t run = Grp::scan(s.waves, mine, &all);
        // (they are of one bin: what lies before it is what lies before them)
        const bool use_k = rules.k < q.a.n, by_list = k_by_list(q, rules);
        const uint64_t each = weight_of_key(tied), before = by_list ? 0 : (use_k ? bins.k_mass_before : bins.p_mass_before);
        uint64_t keep = use_k ? min(all, (uint64_t)rules.k - (by_list ? 0 : bins.k_before)) : all;
        if (rules.p < 1.0f) {
            const double limit = (double)rules.p * (double)(use_k ? before + keep * each : bins.mass);
            uint64_t lo = 0;
            while (lo < keep) {                         // the last one that begins below
                const uint64_t mid = (lo + keep + 1) / 2;
                if (begins_below(true, before + (mid - 1) * each, 0, limit)) lo = mid;
                else keep = mid - 1;
            }
        }
        const uint64_t drawn = kept_weight(distance_of(tied), rules.least);
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const uint64_t inside = min((uint64_t)held_by[i], keep > run ? keep - run : 0);
            if (inside > 0) {
                weight[threadIdx.x * S + i] += drawn * inside;
                if (run + inside == keep) {             // (one segment)
                    found = (int)threadIdx.x * S + i;
                    found_before = run;
                }
            }
            run += held_by[i];
        }
        __syncthreads();
        uint32_t key[E];
        const int64_t from = keys_of(found, key);
        uint64_t ones = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) ones += key[j] == tied ? 1 : 0;
        run = found_before + Grp::scan(s.waves, ones, &all);
        uint64_t mark = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            run += key[j] == tied ? 1 : 0;
            mark = key[j] == tied && run == keep ? (uint64_t)tied << 32 | (uint32_t)(from + j) : mark;
        }
        cut = Grp::most(s, mark);
    } else if (cut_it) {
        const RowBins bins = q.bins[r];
        const bool whole = listed <= (uint32_t)q.list_size;
        const bool near = listed <= kLdsList;
        const uint64_t *const list = q.list + (int64_t)r * q.list_size;
        if (near)
            for (uint32_t i = threadIdx.x; i < listed; i += 1024) held[i] = list[i];        // (a thread reads its own ones)
        // those up to the cut, of one bin (or all)
        auto entries = [&](int bin, auto what) {
            const int64_t n = whole ? (int64_t)listed : q.a.n;
            for (int64_t i = threadIdx.x; i < n; i += 1024) {
                uint64_t at;
                if (near) at = held[i];
                else if (whole) at = list[i];
                else at = (uint64_t)key_of(distance_from(p.top, logit_of(x[i]), rules.inv)) << 32 | (uint32_t)i;
                const uint32_t key = (uint32_t)(at >> 32);
                if (key < kMaskedKey && at <= cut && (bin < 0 || bin_of(key, bins.scale, kLongBins) == bin)) what(at, key);
            }
        };
        // top-k's cut, then top-p's.  (One place that looks for both: twice, the code does not fit the instruction cache.)
        for (int by_mass = rules.k < q.a.n ? 0 : 1; by_mass < (rules.p < 1.0f ? 2 : 1); ++by_mass) {
            int bin = bins.k_bin;
            uint64_t n = bins.k_count, before = bins.k_before;
            double limit = 0.0;
            if (by_mass) {
                uint64_t w = 0;
                if (rules.k < q.a.n) {
                    entries(k_by_list(q, rules) ? -1 : bins.k_bin, [&](uint64_t, uint32_t key) { w += weight_of_key(key); });
                    w = Grp::sum(s, w);
                }
                n = whole ? (uint64_t)listed : (uint64_t)q.a.n;         // (at most)
                bin = -1;
                before = 0;
                if (k_by_list(q, rules)) limit = (double)rules.p * (double)w;
                else {
                    limit = (double)rules.p * (double)(rules.k < q.a.n ? bins.k_mass_before + w : bins.mass);
                    const uint64_t *const mass = q.mass + (int64_t)r * kLongBins;
                    bin = bins.p_first;
                    before = bins.p_mass_before;
                    uint64_t m = before;
                    for (int b = bins.p_first; b <= bins.p_last; ++b) {
                        const uint64_t own = mass[b];
                        if (own > 0 && begins_below(true, m, 0, limit)) { bin = b; before = m; }
                        m += own;
                    }
                }
            }
            cut = Grp::last_below(s, [&](auto what) { entries(bin, what); }, n, by_mass != 0, (uint64_t)rules.k, limit, before);
        }
        // what the list adds to the segments (the row itself, where the list is not whole: everything)
        if (!whole)
            for (int i = threadIdx.x; i < segments; i += 1024) weight[i] = 0;
        __syncthreads();
        entries(-1, [&](uint64_t at, uint32_t key) {
            const uint64_t w = kept_weight(distance_of(key), rules.least);
            if (w) atomicAdd(reinterpret_cast<unsigned long long *>(&weight[(uint32_t)at / (uint32_t)segment]), (unsigned long long)w);
        });
    }
    __syncthreads();
    uint64_t total;
    mine = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) mine += (int)threadIdx.x * S + i < segments ? weight[threadIdx.x * S + i] : 0;
    uint64_t run = Grp::scan(s.waves, mine, &total);
    const double mark = rules.u * (double)total;
    auto beyond = [&](uint64_t v) { return ((double)v > mark) | (v == total); };
    if (beyond(run + mine) && !beyond(run)) {           // (one thread)
        for (int i = threadIdx.x * S; i < segments; ++i) {
            if (beyond(run + weight[i])) {
                found = i;
                found_before = run;
                break;
            }
            run += weight[i];
        }
    }
    __syncthreads();
    uint32_t key[E];
    const int64_t from = keys_of(found, key);
    auto drawn = [&](int j) -> uint64_t {
        return key[j] < kMaskedKey && ((uint64_t)key[j] << 32 | (uint32_t)(from + j)) <= cut ? kept_weight(distance_of(key[j]), rules.least) : 0;
    };
    uint64_t all;
    mine = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) mine += drawn(j);
    run = found_before + Grp::scan(s.waves, mine, &all);
    if (beyond(run + mine) && !beyond(run)) {
        bool open = true;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            run += drawn(j);
            if (open && beyond(run)) {
                open = false;
                q.a.token[row] = (int32_t)(from + j);
                if (q.a.logprob) q.a.logprob[row] = -distance_of(key[j]) - log_of(total);
            }
        }
    }
}

// chunks of a row where so many rows go side by side: 512 workgroups in all, of 4096 to 65,536 entries
int64_t chunk_of(int64_t rows, int64_t n)
{
    const int64_t unit = (int64_t)kLongThreads * kLoad;
    const int64_t pieces = std::max<int64_t>((n + kMostChunk - 1) / kMostChunk, std::min<int64_t>(kMostPieces / rows, n / unit));
    return ((n + pieces - 1) / pieces + unit - 1) / unit * unit;
}

struct LongLayout {
    int64_t rows, chunk, pieces;
    int64_t piece, weight, mass, count, listed, in_bins, list, bins, total;
};
LongLayout long_layout(int64_t rows, int64_t n)
{
    LongLayout L;
    L.rows = std::min(rows, kLongRows);
    L.chunk = chunk_of(L.rows, n);
    L.pieces = (n + L.chunk - 1) / L.chunk;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += align_up(bytes, 256); return here; };
    L.piece = take(L.rows * L.pieces * (int64_t)sizeof(Piece));
    L.weight = take(L.rows * L.pieces * kLongWaves * 8);
    L.mass = take(L.rows * kLongBins * 8);
    L.count = take(L.rows * kLongBins * 4);
    L.listed = take(L.rows * 4);
    L.in_bins = take(L.rows * L.pieces * kLongWaves * (int64_t)sizeof(InBins));
    L.list = take(L.rows * list_of(n) * 8);
    L.bins = take(L.rows * (int64_t)sizeof(RowBins));
    L.total = at;
    return L;
}

template <typename T>
hipError_t launch_long_rows(const SampleArgs &a, char *ws, hipStream_t s)
{
    const LongLayout L = long_layout(a.rows, a.n);
    for (int64_t row0 = 0; row0 < a.rows; row0 += L.rows) {
        LongArgs q;
        q.a = a;
        q.row0 = row0;
        q.rows = (int32_t)std::min(L.rows, a.rows - row0);
        q.chunk = L.chunk;
        q.pieces = (int32_t)L.pieces;
        q.list_size = (int32_t)list_of(a.n);
        q.piece = reinterpret_cast<Piece *>(ws + L.piece);
        q.weight = reinterpret_cast<uint64_t *>(ws + L.weight);
        q.mass = reinterpret_cast<uint64_t *>(ws + L.mass);
        q.count = reinterpret_cast<uint32_t *>(ws + L.count);
        q.listed = reinterpret_cast<uint32_t *>(ws + L.listed);
        q.in_bins = reinterpret_cast<InBins *>(ws + L.in_bins);
        q.list = reinterpret_cast<uint64_t *>(ws + L.list);
        q.bins = reinterpret_cast<RowBins *>(ws + L.bins);
        const dim3 grid((unsigned)q.pieces, (unsigned)q.rows), each((unsigned)q.rows), threads(kLongThreads);
        hipLaunchKernelGGL(long_top_kernel<T>, grid, threads, 0, s, q);
        if (a.top_k || a.top_p) {
            hipLaunchKernelGGL(long_histogram_kernel<T>, grid, threads, 0, s, q);
            hipLaunchKernelGGL(long_bins_kernel, each, threads, 0, s, q);
        }
        hipLaunchKernelGGL(long_weight_kernel<T>, grid, threads, 0, s, q);
        hipLaunchKernelGGL(long_draw_kernel<T>, each, dim3(1024), 0, s, q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_sample(const SampleArgs &a, char *ws, hipStream_t s)
{
    if (a.n <= kThreadRow) return launch_short_rows<T>(a, s);
    if (a.n <= kLaneRow) {
        auto *const kernel = a.n <= 32 ? sample_lanes_kernel<T, 2> : a.n <= 48 ? sample_lanes_kernel<T, 3> : sample_lanes_kernel<T, 4>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + 15) / 16)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    if (a.n <= kGroupRow) return launch_group_rows<T>(a, s);
    return launch_long_rows<T>(a, ws, s);
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int64_t rls_sample_workspace_bytes(int64_t rows, int64_t n_choices)
{
    if (rows < 1 || rows > RLS_MAX_N || n_choices < 1 || n_choices > RLS_MAX_CHOICES) return RLS_ERR_INVALID_ARG;
    return n_choices > kGroupRow ? long_layout(rows, n_choices).total : 0;
}

int32_t rls_sample(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                   const float *uniform_dev, const float *temperature_dev, const int32_t *top_k_dev, const float *top_p_dev,
                   const float *min_p_dev, int32_t *token_dev, float *logprob_dev, void *workspace_dev,
                   int64_t workspace_bytes, void *stream)
{
    if (!logits_dev || !uniform_dev || !token_dev) return RLS_ERR_NULL;
    const int64_t need = rls_sample_workspace_bytes(rows, n_choices);
    if (need < 0) return (int32_t)need;
    if (!is_type(logits_type)) return RLS_ERR_INVALID_ARG;
    if (ld_logits < n_choices) return RLS_ERR_SHAPE;
    if (need > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 256 != 0 || workspace_bytes < need)) return RLS_ERR_WORKSPACE;
    const SampleArgs p{logits_dev, rows, n_choices, ld_logits, uniform_dev, temperature_dev, top_k_dev, top_p_dev, min_p_dev, token_dev, logprob_dev};
    const hipStream_t s = (hipStream_t)stream;
    char *const ws = static_cast<char *>(workspace_dev);
    if (logits_type == RLS_F32) RLS_HIP_TRY(launch_sample<float>(p, ws, s));
    else if (logits_type == RLS_BF16) RLS_HIP_TRY(launch_sample<__bf16>(p, ws, s));
    else RLS_HIP_TRY(launch_sample<_Float16>(p, ws, s));
    return RLS_OK;
}

}  // extern "C"
