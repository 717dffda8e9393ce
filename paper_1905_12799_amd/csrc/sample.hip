// A draw per row of logits with temperature, top-k, top-p and min-p (rls.h gives the rules).
//
// With d = (x - x_max) / temperature every rule but min-p is a cut in the order of descending d, equal ones by index.  -d is
// not negative, so its bits (the key) order like it does; key and index in one word are the entry's place, no two alike, and
// a cut is a place: what lies up to it is kept.  Weights are whole numbers, so their sums do not depend on who adds what.
//
// Reading the logits bounds it, 2 or 4 bytes for a maximum, an exponential and a sum.  What is done with a row goes by its length:
// - up to kThreadRow entries a thread takes a row, in registers, places counted against each other;
// - up to kGroupRow a workgroup of 64 to 1024 threads takes a row, read once into registers, a thread 4 to 32 entries in a row of
//   them.  A cut is found by a histogram over d (counts and weights in LDS) and, in the bin it lies in, by counting the places
//   before each; where a bin holds more than fit the list in LDS, it is cut into bins of places, again and again.
// - longer rows are cut into chunks, a workgroup each; a launch for each of the passes.
#include <algorithm>

#include "element_types.h"
#include "rls_internal.h"

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
    float p, least;                                     // of top-p (1: all), min-p (0: all)
    double u;
};
__device__ inline RowRules rules_of(const SampleArgs &a, int64_t row)
{
    RowRules r{1.0f, a.n, 1.0f, 0.0f, 0.0};
    if (a.top_k) {
        const int32_t k = a.top_k[row];
        if (k >= 1 && k < a.n) r.k = k;
    }
    if (a.temperature) {
        const float t = a.temperature[row];
        if (t > 0.0f) r.inv = 1.0f / t;
        else r.k = 1;
    }
    if (a.top_p && a.top_p[row] < 1.0f) r.p = a.top_p[row];
    if (a.min_p && a.min_p[row] > 0.0f) r.least = a.min_p[row];
    const float u = a.uniform[row];
    if (u > 0.0f) r.u = (double)u;
    return r;
}

// (NaN counts as -infinity)
template <typename T>
__device__ inline float logit_of(T x)
{
    const float v = (float)x;
    return v == v ? v : -INFINITY;
}
__device__ inline float scaled_logit(float x, float top, float inv)
{
    const float gap = x - top;
    return x == top ? 0.0f : (gap == -INFINITY ? -INFINITY : gap * inv);
}
__device__ inline uint32_t key_of(float d) { return __float_as_uint(d) & 0x7fffffffu; }
__device__ inline float distance_of(uint32_t key) { return __uint_as_float(key); }       // -d

// weight of an entry: exp(d) in multiples of 2^-38 (adding 1.5 * 2^14 leaves the whole number in the low bits of a double)
__device__ inline uint64_t weight_of(float e)
{
    constexpr double kMagic = 1.5 * 16384.0;
    return (uint64_t)(__double_as_longlong((double)e + kMagic) - __double_as_longlong(kMagic));
}
__device__ inline uint64_t weight_of_key(uint32_t key) { return weight_of(expf(-distance_of(key))); }
// whether an entry with so many entries, or so much weight, before it is inside top-k, or top-p (the first one always is)
__device__ inline bool begins_below(bool by_mass, uint64_t count, uint64_t mass, uint64_t k, double limit)
{
    return by_mass ? mass == 0 || (double)mass < limit : count < k;
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
    float d[V], e[V];
    uint64_t w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        d[i] = scaled_logit(l[i], top, r.inv);
        e[i] = expf(d[i]);
        w[i] = d[i] > -INFINITY ? weight_of(e[i]) : 0;
    }
    if (r.k < n || r.p < 1.0f) {
        uint64_t before[V], total = 0;                  // weight of what comes before an entry, top-k applied
        uint32_t in = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            int rank = 0;
            before[i] = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool first = (d[j] > d[i]) | ((d[j] == d[i]) & (j < i));
                rank += first;
                before[i] += first ? w[j] : 0;
            }
            // (where an entry is inside top-k so is everything before it)
            in |= (rank < r.k ? 1u : 0u) << i;
            total += rank < r.k ? w[i] : 0;
        }
        const double limit = (double)r.p * (double)total;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            // (a selection, no branches: hipcc 7.2 loses the assignment of an element of an array in registers behind nested conditions)
            const bool out = ((in >> i & 1u) == 0) | ((r.p < 1.0f) & (before[i] > 0) & ((double)before[i] >= limit));
            w[i] = out ? 0 : w[i];
        }
    }
    uint64_t total = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = (e[i] < r.least) & (d[i] != 0.0f) ? 0 : w[i];
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
        d_token = here ? d[i] : d_token;
    }
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = d_token - log_of(total);
}

// ---- a workgroup's tools --------------------------------------------------------------------------

template <int NT>
struct Group {
    static constexpr int kWaves = NT / 64;
    static constexpr int kBins = NT == 64 ? 256 : 1024;
    static constexpr int kList = NT == 64 ? 256 : (NT < 1024 ? 512 : 1024);    // places that are counted against each other
    static constexpr int kBinsOfThread = kBins / NT;

    struct Shared {
        uint64_t mass[kBins];
        uint32_t count[kBins];
        uint64_t place[kList], weight[kList];
        uint64_t wave_a[kWaves], wave_b[kWaves];
        uint64_t found_mass;
        uint32_t found_bin, found_n, found_count, listed;
    };

    static __device__ inline void sync()
    {
        if constexpr (NT == 64) __builtin_amdgcn_wave_barrier();
        __syncthreads();
    }
    // reductions and scans over the workgroup; the results are the same in every thread
    template <typename F>
    static __device__ inline uint64_t reduce(Shared &s, uint64_t x, F join)
    {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) x = join(x, (uint64_t)__shfl_xor((unsigned long long)x, off, 64));
        if constexpr (NT > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s.wave_a[threadIdx.x >> 6] = x;
            __syncthreads();
            x = s.wave_a[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) x = join(x, s.wave_a[w]);
        }
        return x;
    }
    static __device__ inline uint64_t sum(Shared &s, uint64_t x)
    {
        return reduce(s, x, [](uint64_t a, uint64_t b) { return a + b; });
    }
    static __device__ inline uint64_t most(Shared &s, uint64_t x)
    {
        return reduce(s, x, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    }
    static __device__ inline float most_float(Shared &s, float x)
    {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
        if constexpr (NT > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s.wave_a[threadIdx.x >> 6] = __float_as_uint(x);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) x = fmaxf(x, __uint_as_float((uint32_t)s.wave_a[w]));
        }
        return x;
    }
    // what the threads before this one have (and the sum of all)
    static __device__ inline uint64_t scan(Shared &s, uint64_t x, uint64_t *total)
    {
        const int lane = threadIdx.x & 63;
        uint64_t run = x;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint64_t o = __shfl_up((unsigned long long)run, off, 64);
            if (lane >= off) run += o;
        }
        if constexpr (NT == 64) {
            *total = __shfl((unsigned long long)run, 63, 64);
            return run - x;
        } else {
            const int wave = threadIdx.x >> 6;
            __syncthreads();
            if (lane == 63) s.wave_b[wave] = run;
            __syncthreads();
            uint64_t before = 0, all = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint64_t v = s.wave_b[w];
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
    // The last bin whose entries begin below: fewer than k entries before it, or less weight than `limit`, of which so many and so much come
    // before all bins.  Leaves bin, its entries, and entries and weight before it in s.
    static __device__ inline void find_bin(Shared &s, bool by_mass, uint64_t k, double limit, uint64_t base_count, uint64_t base_mass)
    {
        sync();
        uint64_t count = 0, mass = 0, all;
#pragma unroll
        for (int b = 0; b < kBinsOfThread; ++b) {
            count += s.count[threadIdx.x * kBinsOfThread + b];
            mass += s.mass[threadIdx.x * kBinsOfThread + b];
        }
        const uint64_t count_before = base_count + scan(s, count, &all), mass_before = base_mass + scan(s, mass, &all);
        if (threadIdx.x == 0) s.found_bin = 0;
        sync();
        int mine = -1;
        uint64_t c = count_before, m = mass_before;
#pragma unroll
        for (int b = 0; b < kBinsOfThread; ++b) {
            const uint32_t n = s.count[threadIdx.x * kBinsOfThread + b];
            if (n > 0 && begins_below(by_mass, c, m, k, limit)) mine = threadIdx.x * kBinsOfThread + b;
            c += n;
            m += s.mass[threadIdx.x * kBinsOfThread + b];
        }
        if (mine >= 0) atomicMax(&s.found_bin, (uint32_t)mine);
        sync();
        if ((int)(s.found_bin / kBinsOfThread) == (int)threadIdx.x) {
            c = count_before;
            m = mass_before;
#pragma unroll
            for (int b = 0; b < kBinsOfThread; ++b) {
                if (threadIdx.x * kBinsOfThread + b == s.found_bin) {
                    s.found_n = s.count[s.found_bin];
                    s.found_count = (uint32_t)c;
                    s.found_mass = m;
                }
                c += s.count[threadIdx.x * kBinsOfThread + b];
                m += s.mass[threadIdx.x * kBinsOfThread + b];
            }
        }
        sync();
    }
    // Among the n entries that `visit` hands to a function of place and key, the last place that begins below (see find_bin).  Where they fit the
    // list they are counted against each other; more are cut into bins of places first, again and again.
    template <typename Visit>
    static __device__ inline uint64_t last_below(Shared &s, Visit visit, uint64_t n, bool by_mass, uint64_t k, double limit, uint64_t count, uint64_t mass)
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
            find_bin(s, by_mass, k, limit, count, mass);
            lo += (uint64_t)s.found_bin << shift;
            const uint64_t end = lo + ((1ull << shift) - 1);
            hi = end < hi ? end : hi;
            n = s.found_n;
            count = s.found_count;
            mass = s.found_mass;
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
        for (uint32_t i = threadIdx.x; i < listed; i += NT) {
            const uint64_t at = s.place[i];
            uint64_t c = count, m = mass;
            for (uint32_t o = 0; o < listed; ++o) {
                const bool first = s.place[o] < at;
                c += first;
                m += first ? s.weight[o] : 0;
            }
            if (begins_below(by_mass, c, m, k, limit)) cut = cut > at ? cut : at;
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
        auto in_bin = [&](int bin, bool by_mass, double limit, uint64_t n, uint64_t c, uint64_t m) {
            return last_below(s, [&](auto what) {
                x.forget();
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (x.there(j) && bin_of(x.key[j], scale, kBins) == bin && x.upto(j, cut)) what(x.place(j), x.key[j]);
                    pace(j);
                }
            }, n, by_mass, k, limit, c, m);
        };
        int p_bin = 0;
        uint64_t n, c, m;
        if (use_k) {
            find_bin(s, false, k, 0.0, 0, 0);
            const int bin = (int)s.found_bin;
            n = s.found_n, c = s.found_count;
            const bool crowded = n > kList;
            cut = in_bin(bin, false, 0.0, n, c, 0);
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
            find_bin(s, true, 0, limit, 0, 0);
            p_bin = (int)s.found_bin;
            n = s.found_n, m = s.found_mass;
            cut = in_bin(p_bin, true, limit, n, 0, m);
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
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < E; ++j) top = fmaxf(top, l[j]);
        top = Grp::most_float(s, top);
        if (top == -INFINITY) {
            if (threadIdx.x == 0) no_draw(a, row);
            continue;
        }
        const RowRules r = rules_of(a, row);
        typename Grp::template Entries<E> entry;
        entry.first = (uint32_t)first;
        float widest = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float d = scaled_logit(l[j], top, r.inv);
            entry.key[j] = key_of(d);
            if (entry.there(j)) widest = fmaxf(widest, -d);
        }
        uint64_t cut = ~0ull;
        if (r.k < n || r.p < 1.0f)
            cut = Grp::cut_of(s, entry, Grp::most_float(s, widest), (uint64_t)r.k, r.k < n, r.p, r.p < 1.0f);
        auto weight = [&](int j) -> uint64_t {
            if (!entry.there(j) || !entry.upto(j, cut)) return 0;
            const float e = expf(-distance_of(entry.key[j]));
            return e < r.least && entry.key[j] != 0 ? 0 : weight_of(e);
        };
        uint64_t mine = 0, total;
        entry.forget();
#pragma unroll
        for (int j = 0; j < E; ++j) {
            mine += weight(j);
            Grp::pace(j);
        }
        uint64_t run = Grp::scan(s, mine, &total);
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

constexpr int64_t kGroupRow = 32768;
constexpr int64_t kMostGroups = 1 << 20;           // (of a launch, which ends at 2^32 threads)

template <typename T>
hipError_t launch_group_rows(const SampleArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows < kMostGroups ? a.rows : kMostGroups));
    if (a.n <= 256) hipLaunchKernelGGL((sample_row_kernel<T, 64, 4>), grid, dim3(64), 0, s, a);
    else if (a.n <= 1024) hipLaunchKernelGGL((sample_row_kernel<T, 64, 16>), grid, dim3(64), 0, s, a);
    else if (a.n <= 4096) hipLaunchKernelGGL((sample_row_kernel<T, 256, 16>), grid, dim3(256), 0, s, a);
    else if (a.n <= 16384) hipLaunchKernelGGL((sample_row_kernel<T, 1024, 16>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((sample_row_kernel<T, 1024, 32>), grid, dim3(1024), 0, s, a);
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

// Rows are cut into chunks, a workgroup each, and a batch of rows goes through launches: maxima; where a row has top-k or top-p a histogram, the
// entries of the bins that its cuts lie in as a list, and the cuts; the chunks' weights; the draw.  What a launch needs of the row's other
// chunks it finds in the workspace.
constexpr int kLongThreads = 512;
constexpr int kLongBins = 2048;
constexpr int kLongList = 16384;
constexpr int kLongStage = 1024;                        // places a workgroup collects before it goes to the row's list one by one
constexpr int64_t kLongRows = 256;                      // of a batch
constexpr int kMostPieces = 512;                        // chunks of a row
constexpr int kLoad = 8;                                // entries a thread takes in a row

struct Piece {
    float top, low;                                     // the largest, and the smallest that is not masked
    uint32_t at;                                        // where the largest is first
};
struct RowBins {                                        // where a row's cuts lie
    int32_t k_bin, p_first, p_last;                     // top-k's bin; top-p's is one of these, which depends on what top-k keeps of its own
    uint32_t k_count, k_before;
    uint64_t k_mass_before, p_mass_before;              // weight before k_bin, p_first
    float top, scale;
    uint64_t cut;
};
struct LongArgs {
    SampleArgs a;
    int64_t row0, chunk;
    int32_t rows, pieces;
    Piece *piece;                                       // [rows][pieces]
    uint64_t *weight;                                   // [rows][pieces]
    uint64_t *mass;                                     // [rows][kLongBins]
    uint32_t *count, *listed;                           // [rows][kLongBins], [rows]
    uint64_t *list;                                     // [rows][kLongList]
    RowBins *bins;                                      // [rows]
};

template <typename T, typename F>
__device__ inline void visit_chunk(const T *x, int64_t begin, int64_t end, int threads, F what)
{
    for (int64_t i = begin + (int64_t)threadIdx.x * kLoad; i < end; i += (int64_t)threads * kLoad) {
        if (i + kLoad <= end) {
            T v[kLoad];
            __builtin_memcpy(v, x + i, sizeof(v));
#pragma unroll
            for (int j = 0; j < kLoad; ++j) what(logit_of(v[j]), i + j);
        } else {
            for (int64_t j = i; j < end; ++j) what(logit_of(x[j]), j);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_top_kernel(LongArgs q)
{
    __shared__ float tops[kLongThreads / 64], lows[kLongThreads / 64];
    __shared__ uint32_t ats[kLongThreads / 64];
    const int piece = blockIdx.x, r = blockIdx.y;
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    float top = -INFINITY, low = INFINITY;
    uint32_t at = ~0u;
    visit_chunk(x, begin, end, kLongThreads, [&](float v, int64_t i) {
        if (v > top) { top = v; at = (uint32_t)i; }     // (a thread's indices ascend)
        if (v > -INFINITY) low = fminf(low, v);
    });
    auto join = [&](float t, float l, uint32_t i) {
        if (t > top || (t == top && i < at)) { top = t; at = i; }
        low = fminf(low, l);
    };
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) join(__shfl_xor(top, off, 64), __shfl_xor(low, off, 64), (uint32_t)__shfl_xor((int)at, off, 64));
    if ((threadIdx.x & 63) == 0) { tops[threadIdx.x >> 6] = top; lows[threadIdx.x >> 6] = low; ats[threadIdx.x >> 6] = at; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kLongThreads / 64; ++w) join(tops[w], lows[w], ats[w]);
        q.piece[(int64_t)r * q.pieces + piece] = Piece{top, low, at};
        if (piece == 0) q.listed[r] = 0;
    }
    // the row's histogram is cleared by its workgroups together
    for (int b = piece * kLongThreads + threadIdx.x; b < kLongBins; b += q.pieces * kLongThreads) {
        q.count[(int64_t)r * kLongBins + b] = 0;
        q.mass[(int64_t)r * kLongBins + b] = 0;
    }
}

// The whole row's largest entry, the first place it is at, and the smallest that is not masked
template <int NT>
__device__ inline Piece row_top(const LongArgs &q, int r, Piece *lds)
{
    Piece p{-INFINITY, INFINITY, ~0u};
    auto join = [&](const Piece &o) {
        if (o.top > p.top || (o.top == p.top && o.at < p.at)) { p.top = o.top; p.at = o.at; }
        p.low = fminf(p.low, o.low);
    };
    for (int i = threadIdx.x; i < q.pieces; i += NT) join(q.piece[(int64_t)r * q.pieces + i]);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1)
        join(Piece{__shfl_xor(p.top, off, 64), __shfl_xor(p.low, off, 64), (uint32_t)__shfl_xor((int)p.at, off, 64)});
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = p;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) join(lds[w]);
    __syncthreads();
    return p;
}

// whether a row's cut has to be looked for (a single entry, its largest, is known from the maxima)
__device__ inline bool cuts(const LongArgs &q, const RowRules &r, float top) { return top > -INFINITY && r.k != 1 && (r.k < q.a.n || r.p < 1.0f); }

template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_histogram_kernel(LongArgs q)
{
    __shared__ uint64_t mass[kLongBins];
    __shared__ uint32_t count[kLongBins];
    __shared__ Piece lds[kLongThreads / 64];
    const int piece = blockIdx.x, r = blockIdx.y;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const Piece p = row_top<kLongThreads>(q, r, lds);
    if (!cuts(q, rules, p.top)) return;
    const float scale = bin_scale(-scaled_logit(p.low, p.top, rules.inv), kLongBins);
    if (piece == 0 && threadIdx.x == 0) {
        q.bins[r].top = p.top;
        q.bins[r].scale = scale;
    }
    for (int b = threadIdx.x; b < kLongBins; b += kLongThreads) { count[b] = 0; mass[b] = 0; }
    __syncthreads();
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    const bool use_p = rules.p < 1.0f;
    visit_chunk(x, begin, end, kLongThreads, [&](float v, int64_t) {
        const uint32_t key = key_of(scaled_logit(v, p.top, rules.inv));
        if (key >= kMaskedKey) return;
        const int b = bin_of(key, scale, kLongBins);
        atomicAdd(&count[b], 1u);
        if (use_p) atomicAdd(reinterpret_cast<unsigned long long *>(&mass[b]), (unsigned long long)weight_of_key(key));
    });
    __syncthreads();
    for (int b = threadIdx.x; b < kLongBins; b += kLongThreads)
        if (count[b]) {
            atomicAdd(&q.count[(int64_t)r * kLongBins + b], count[b]);
            if (use_p && mass[b]) atomicAdd(reinterpret_cast<unsigned long long *>(&q.mass[(int64_t)r * kLongBins + b]), (unsigned long long)mass[b]);
        }
}

// From the row's histogram the bins that its cuts lie in; then the entries of a chunk in these bins.
template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_list_kernel(LongArgs q)
{
    using Grp = Group<kLongThreads>;
    __shared__ typename Grp::Shared s;
    __shared__ uint64_t stage[kLongStage];
    __shared__ uint32_t staged, base;
    __shared__ int32_t bin_k, bin_first, bin_last;
    constexpr int B = kLongBins / kLongThreads;
    const int piece = blockIdx.x, r = blockIdx.y;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    float top = -INFINITY;
    for (int i = 0; i < q.pieces; i += 64) {            // (a wave's worth at a time)
        const int at = i + (threadIdx.x & 63);
        top = fmaxf(top, at < q.pieces ? q.piece[(int64_t)r * q.pieces + at].top : -INFINITY);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (!cuts(q, rules, top)) return;
    const float scale = q.bins[r].scale;
    uint32_t count[B];
    uint64_t mass[B], n = 0, w = 0, all_n, all_w;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        count[b] = q.count[(int64_t)r * kLongBins + threadIdx.x * B + b];
        mass[b] = q.mass[(int64_t)r * kLongBins + threadIdx.x * B + b];
        n += count[b];
        w += mass[b];
    }
    const uint64_t n_before = Grp::scan(s, n, &all_n), w_before = Grp::scan(s, w, &all_w);
    if (threadIdx.x == 0) { bin_k = -1; bin_first = bin_last = -1; staged = 0; }
    __syncthreads();
    // the last bin that begins below, for `below` of the entries and the weight before it
    auto last_bin = [&](int32_t *found, auto below) {
        uint64_t c = n_before, m = w_before;
        int mine = -1;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (count[b] > 0 && below(c, m)) mine = threadIdx.x * B + b;
            c += count[b];
            m += mass[b];
        }
        if (mine >= 0) atomicMax(found, mine);
        __syncthreads();
    };
    // weight that top-k keeps, at least and at most
    uint64_t least = all_w, most = all_w;
    RowBins *const out = &q.bins[r];
    // a bin's count, and entries and weight before it, by the thread that has it
    auto of_bin = [&](int bin, auto what) {
        uint64_t c = n_before, m = w_before;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if ((int)threadIdx.x * B + b == bin) what(count[b], mass[b], c, m);
            c += count[b];
            m += mass[b];
        }
    };
    if (rules.k < q.a.n) {
        last_bin(&bin_k, [&](uint64_t c, uint64_t) { return c < (uint64_t)rules.k; });
        of_bin(bin_k, [&](uint32_t c, uint64_t m, uint64_t c0, uint64_t m0) {
            s.place[0] = m0;
            s.place[1] = m0 + m;
            if (piece == 0) {
                out->k_count = c;
                out->k_before = (uint32_t)c0;
                out->k_mass_before = m0;
            }
        });
        __syncthreads();
        least = s.place[0];
        most = s.place[1];
    }
    if (rules.p < 1.0f) {
        last_bin(&bin_first, [&](uint64_t c, uint64_t m) { return begins_below(true, c, m, 0, (double)rules.p * (double)least); });
        last_bin(&bin_last, [&](uint64_t c, uint64_t m) { return begins_below(true, c, m, 0, (double)rules.p * (double)most); });
        if (piece == 0) of_bin(bin_first, [&](uint32_t, uint64_t, uint64_t, uint64_t m0) { out->p_mass_before = m0; });
    }
    const int k_bin = bin_k, p_first = bin_first, p_last = bin_last;
    if (piece == 0 && threadIdx.x == 0) {
        out->k_bin = k_bin;
        out->p_first = p_first;
        out->p_last = p_last;
    }
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    visit_chunk(x, begin, end, kLongThreads, [&](float v, int64_t i) {
        const uint32_t key = key_of(scaled_logit(v, top, rules.inv));
        if (key >= kMaskedKey) return;
        const int b = bin_of(key, scale, kLongBins);
        if (b != k_bin && (b < p_first || b > p_last || p_first < 0)) return;
        const uint64_t place = (uint64_t)key << 32 | (uint32_t)i;
        const uint32_t at = atomicAdd(&staged, 1u);
        if (at < kLongStage) stage[at] = place;
        else {
            const uint32_t to = atomicAdd(&q.listed[r], 1u);
            if (to < kLongList) q.list[(int64_t)r * kLongList + to] = place;
        }
    });
    __syncthreads();
    const uint32_t own = staged < kLongStage ? staged : kLongStage;
    if (threadIdx.x == 0) base = atomicAdd(&q.listed[r], own);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < own; i += kLongThreads)
        if (base + i < kLongList) q.list[(int64_t)r * kLongList + base + i] = stage[i];
}

// The cuts, from the list, or from the row itself where its bins hold more entries than the list.
template <typename T>
__global__ void __launch_bounds__(1024) long_cut_kernel(LongArgs q)
{
    using Grp = Group<1024>;
    __shared__ typename Grp::Shared s;
    __shared__ Piece lds[1024 / 64];
    const int r = blockIdx.x;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const Piece p = row_top<1024>(q, r, lds);
    if (!cuts(q, rules, p.top)) return;
    const RowBins bins = q.bins[r];
    const uint32_t listed = q.listed[r];
    const uint64_t *const list = q.list + (int64_t)r * kLongList;
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    uint64_t cut = ~0ull;
    auto entries_of = [&](int bin) {
        return [&, bin](auto what) {
            if (listed <= kLongList) {
                for (uint32_t i = threadIdx.x; i < listed; i += 1024) {
                    const uint64_t at = list[i];
                    const uint32_t key = (uint32_t)(at >> 32);
                    if (at <= cut && bin_of(key, bins.scale, kLongBins) == bin) what(at, key);
                }
            } else {
                visit_chunk(x, 0, q.a.n, 1024, [&](float v, int64_t i) {
                    const uint32_t key = key_of(scaled_logit(v, p.top, rules.inv));
                    const uint64_t at = (uint64_t)key << 32 | (uint32_t)i;
                    if (key < kMaskedKey && at <= cut && bin_of(key, bins.scale, kLongBins) == bin) what(at, key);
                });
            }
        };
    };
    const uint32_t *const count = q.count + (int64_t)r * kLongBins;
    const uint64_t *const mass = q.mass + (int64_t)r * kLongBins;
    uint64_t kept = 0;
    if (rules.k < q.a.n) {
        cut = Grp::last_below(s, entries_of(bins.k_bin), bins.k_count, false, (uint64_t)rules.k, 0.0, bins.k_before, 0);
        if (rules.p < 1.0f) {
            uint64_t w = 0;
            entries_of(bins.k_bin)([&](uint64_t, uint32_t key) { w += weight_of_key(key); });
            kept = bins.k_mass_before + Grp::sum(s, w);
        }
    } else {
        uint64_t w = 0;
        for (int b = threadIdx.x; b < kLongBins; b += 1024) w += mass[b];
        kept = Grp::sum(s, w);
    }
    if (rules.p < 1.0f) {
        const double limit = (double)rules.p * (double)kept;
        int bin = bins.p_first;
        uint64_t before = bins.p_mass_before, m = before;
        for (int b = bins.p_first; b <= bins.p_last; ++b) {
            if (count[b] > 0 && begins_below(true, 0, m, 0, limit)) { bin = b; before = m; }
            m += mass[b];
        }
        cut = Grp::last_below(s, entries_of(bin), count[bin], true, 0, limit, 0, before);
    }
    if (threadIdx.x == 0) q.bins[r].cut = cut;
}

// what an entry adds to the draw
__device__ inline uint64_t drawn_weight(float v, int64_t i, float top, const RowRules &rules, uint64_t cut, uint32_t *key_out)
{
    const float d = scaled_logit(v, top, rules.inv);
    const uint32_t key = key_of(d);
    *key_out = key;
    if (key >= kMaskedKey || ((uint64_t)key << 32 | (uint32_t)i) > cut) return 0;
    const float e = expf(d);
    return e < rules.least && key != 0 ? 0 : weight_of(e);
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) long_weight_kernel(LongArgs q)
{
    __shared__ Piece lds[kLongThreads / 64];
    __shared__ uint64_t sums[kLongThreads / 64];
    const int piece = blockIdx.x, r = blockIdx.y;
    const RowRules rules = rules_of(q.a, q.row0 + r);
    const Piece p = row_top<kLongThreads>(q, r, lds);
    if (!(p.top > -INFINITY) || rules.k == 1) return;
    const uint64_t cut = cuts(q, rules, p.top) ? q.bins[r].cut : ~0ull;
    const T *const x = static_cast<const T *>(q.a.logits) + (q.row0 + r) * q.a.ld;
    const int64_t begin = piece * q.chunk, end = min(q.a.n, begin + q.chunk);
    uint64_t w = 0;
    uint32_t key;
    visit_chunk(x, begin, end, kLongThreads, [&](float v, int64_t i) { w += drawn_weight(v, i, p.top, rules, cut, &key); });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) w += __shfl_xor((unsigned long long)w, off, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = w;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kLongThreads / 64; ++i) w += sums[i];
        q.weight[(int64_t)r * q.pieces + piece] = w;
    }
}

template <typename T>
__global__ void __launch_bounds__(1024) long_draw_kernel(LongArgs q)
{
    using Grp = Group<1024>;
    __shared__ typename Grp::Shared s;
    __shared__ Piece lds[1024 / 64];
    __shared__ int found;
    __shared__ uint64_t found_before;
    const int r = blockIdx.x;
    const int64_t row = q.row0 + r;
    const RowRules rules = rules_of(q.a, row);
    const Piece p = row_top<1024>(q, r, lds);
    if (!(p.top > -INFINITY) || rules.k == 1) {
        if (threadIdx.x == 0) {
            if (p.top > -INFINITY) {
                q.a.token[row] = (int32_t)p.at;
                if (q.a.logprob) q.a.logprob[row] = 0.0f;
            } else no_draw(q.a, row);
        }
        return;
    }
    const uint64_t cut = cuts(q, rules, p.top) ? q.bins[r].cut : ~0ull;
    uint64_t total;
    const uint64_t w = (int)threadIdx.x < q.pieces ? q.weight[(int64_t)r * q.pieces + threadIdx.x] : 0;
    uint64_t run = Grp::scan(s, w, &total);
    const double mark = rules.u * (double)total;
    auto beyond = [&](uint64_t v) { return (double)v > mark || v == total; };
    if (beyond(run + w) && !beyond(run)) {              // (one chunk)
        found = (int)threadIdx.x;
        found_before = run;
    }
    __syncthreads();
    // the chunk, a part per thread in the order of the entries
    const T *const x = static_cast<const T *>(q.a.logits) + row * q.a.ld;
    const int64_t begin = found * q.chunk, end = min(q.a.n, begin + q.chunk), part = (end - begin + 1023) / 1024;
    const int64_t from = min(end, begin + part * threadIdx.x), to = min(end, from + part);
    uint64_t mine = 0, all;
    uint32_t key;
    for (int64_t i = from; i < to; ++i) mine += drawn_weight(logit_of(x[i]), i, p.top, rules, cut, &key);
    run = found_before + Grp::scan(s, mine, &all);
    if (beyond(run + mine) && !beyond(run)) {
        for (int64_t i = from; i < to; ++i) {
            run += drawn_weight(logit_of(x[i]), i, p.top, rules, cut, &key);
            if (beyond(run)) {
                q.a.token[row] = (int32_t)i;
                if (q.a.logprob) q.a.logprob[row] = -distance_of(key) - log_of(total);
                break;
            }
        }
    }
}

// chunks of a row where so many rows go side by side: 512 workgroups in all, of 4096 to 65,536 entries
int64_t chunk_of(int64_t rows, int64_t n)
{
    const int64_t unit = (int64_t)kLongThreads * kLoad;
    const int64_t pieces = std::max<int64_t>((n + 65535) / 65536, std::min<int64_t>(kMostPieces / rows, n / unit));
    return ((n + pieces - 1) / pieces + unit - 1) / unit * unit;
}

struct LongLayout {
    int64_t rows, chunk, pieces;
    int64_t piece, weight, mass, count, listed, list, bins, total;
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
    L.weight = take(L.rows * L.pieces * 8);
    L.mass = take(L.rows * kLongBins * 8);
    L.count = take(L.rows * kLongBins * 4);
    L.listed = take(L.rows * 4);
    L.list = take(L.rows * kLongList * 8);
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
        q.piece = reinterpret_cast<Piece *>(ws + L.piece);
        q.weight = reinterpret_cast<uint64_t *>(ws + L.weight);
        q.mass = reinterpret_cast<uint64_t *>(ws + L.mass);
        q.count = reinterpret_cast<uint32_t *>(ws + L.count);
        q.listed = reinterpret_cast<uint32_t *>(ws + L.listed);
        q.list = reinterpret_cast<uint64_t *>(ws + L.list);
        q.bins = reinterpret_cast<RowBins *>(ws + L.bins);
        const dim3 grid((unsigned)q.pieces, (unsigned)q.rows), each((unsigned)q.rows), threads(kLongThreads);
        hipLaunchKernelGGL(long_top_kernel<T>, grid, threads, 0, s, q);
        if (a.top_k || a.top_p) {
            hipLaunchKernelGGL(long_histogram_kernel<T>, grid, threads, 0, s, q);
            hipLaunchKernelGGL(long_list_kernel<T>, grid, threads, 0, s, q);
            hipLaunchKernelGGL(long_cut_kernel<T>, each, dim3(1024), 0, s, q);
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
