// Log-probabilities of given entries per row of logits, with the entropy and the best alternatives; the divergence from a teacher's best
// entries; the gradients of both by the logits (rls.h gives the formulas).
//
// One pass over a row keeps, thread by thread, the largest logit so far, the sum of 2^d2 and the sum of 2^d2 d2 beside it, with
// d2 = (x - largest) log2(e) / temperature; a larger logit scales both down.  From the three come the logarithm of the sum, the
// entropy and every entry's log-probability.  An entry that does not count (-infinity, NaN) has d2 = -200, whose power is 0 in fp32: the
// maximum that ends d2 there also takes NaN to it, so nothing is asked about an entry.  +infinity counts as the largest number.
//
// The best alternatives need no order of the row.  An entry's place is its logit's bits, ordered, with the index below them, no two
// alike.  The best places of the threads are known after the pass; at least `top` of them are at or above a threshold between them, and what is
// at or above it lies with those few threads, which read their part again and list it.
//
// Reading the logits bounds the forward pass, reading and writing them the backward one: 4096 x 50021 in bf16 forward 89 us (4.6 TB/s), 8192 x 32001 in bf16
// backward 211 (5.0 TB/s; a copy of 2 GiB 4.9), 2048 x 128003 with 64 entries of a teacher 216 (4.9).  Where there is little to read it is dependent steps: 524288 x 3
// in fp32 5 us forward and 5 backward, 524288 x 20 33 and 41 (bf16 46 and 65: fewer lanes have entries), 64 x 128003 in bf16 with 20 alternatives 18 and 8 (7 and 4 without).
#include <algorithm>

#include "element_types.h"
#include "rls_internal.h"
#include "wave.h"

namespace rls {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLeast = -200.0f;                        // of d2: 2^-200 is 0
constexpr float kLargest = 3.4028234663852886e38f;
constexpr int kThreadRow = 16;                           // entries that a thread takes by itself
constexpr int kWaveRow = 1024;                           // a wave, or 16 lanes
constexpr int kListed = 4096;                            // places that a workgroup's list holds
constexpr int kRanked = 256;                             // of them that are counted against each other at once

struct RowArgs {
    const void *logits;
    int64_t row0, rows, n, ld;                           // rows row0 .. rows - 1 by this launch
    const float *temperature;
    const int32_t *token;                                // logprobs: [rows]; distill: [rows][k]
    float *logprob, *entropy, *norm;                     // distill: logprob is the loss
    int32_t top;
    float *top_logprob;
    int32_t *top_token;
    const void *teacher;                                 // distill: [rows][k]
    int32_t k, teacher_type;
    // rows in pieces
    int32_t pieces;
    int64_t piece;
    float *part;                                         // [rows][pieces][4]
    uint64_t *best;                                      // [rows][pieces][top]
};

// 1 / temperature: 1 without one; at most 2e38, so that log2(e) times it is a number
__device__ inline float inverse_of(const float *temperature, int64_t row)
{
    if (!temperature) return 1.0f;
    const float t = temperature[row];
    return t > 0.0f ? fminf(1.0f / t, 2e38f) : 1.0f;
}
// (NaN stays NaN until a distance is taken)
template <typename T>
__device__ inline float logit_of(T x)
{
    const float v = (float)x;
    return v > kLargest ? kLargest : v;
}
__device__ inline float power_of(float d2) { return __builtin_amdgcn_exp2f(d2); }
__device__ inline float distance2(float x, float top, float c) { return fmaxf((x - top) * c, kLeast); }

// 16 bytes of a row, which may begin at any element
template <typename T>
struct Pack {
    static constexpr int N = 16 / sizeof(T);
    T x[N];
};
template <typename T>
__device__ inline Pack<T> load_pack(const T *p)
{
    Pack<T> v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T>
__device__ inline void store_pack(T *p, const Pack<T> &v)
{
    __builtin_memcpy(p, &v, 16);
}

// Place of an entry in the order of falling logits, equal ones by rising index; larger is earlier, 0 is none
__device__ inline uint64_t place_of(float x, uint32_t index)
{
    if (!(x > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(x + 0.0f);        // (-0 and 0 are equal)
    return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~index;
}
__device__ inline float logit_at(uint64_t place)
{
    const uint32_t b = (uint32_t)(place >> 32);
    return __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ inline uint32_t index_at(uint64_t place) { return ~(uint32_t)place; }

// What a thread, a piece or a row has seen
struct Seen {
    float top = -INFINITY, sum = 0.0f, sum2 = 0.0f;      // sum2: of 2^d2 d2

    __device__ void raise(float to, float c)             // to >= top
    {
        const float d2 = distance2(top, to, c), f = power_of(d2);
        sum2 = f * fmaf(sum, d2, sum2);
        sum *= f;
        top = to;
    }
    __device__ void add(float x, float c)
    {
        const float d2 = distance2(x, top, c), e = power_of(d2);
        sum += e;
        sum2 = fmaf(e, d2, sum2);
    }
    __device__ float log_sum() const { return sum > 0.0f ? logf(sum) : 0.0f; }
    __device__ float entropy() const { return sum > 0.0f ? fmaxf(logf(sum) - sum2 * kLn2 / sum, 0.0f) : 0.0f; }
    __device__ float logprob(float x, float inv, float log) const
    {
        return x > -INFINITY && top > -INFINITY ? (x - top) * inv - log : -INFINITY;
    }
};
__device__ inline Seen wave_join(Seen v, float c)
{
    v.raise(wave_max(v.top), c);
    const auto plus = [](float a, float b) { return a + b; };
    v.sum = wave_reduce(v.sum, 0.0f, plus);
    v.sum2 = wave_reduce(v.sum2, 0.0f, plus);
    return v;
}

// over the lanes that take a row together, 16 or all 64 of a wave; the same in each of them
template <int L, typename T, typename F>
__device__ inline T lanes_reduce(T x, T none, F join)
{
    return L == 16 ? row_reduce(x, join) : wave_reduce(x, none, join);
}
template <int L>
__device__ inline float lanes_max(float x)
{
    return lanes_reduce<L>(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ inline float lanes_sum(float x)
{
    return lanes_reduce<L>(x, 0.0f, [](float a, float b) { return a + b; });
}

// NT threads that take a row together: a wave by itself, or a workgroup
template <int NT>
struct Team {
    static constexpr int kWaves = NT / 64;
    struct Shared {
        float top[kWaves], sum[kWaves], sum2[kWaves];
        uint32_t count[2][kWaves];
        uint32_t listed;
    };
    static __device__ int tid() { return NT == 64 ? threadIdx.x & 63 : threadIdx.x; }
    static __device__ void sync()
    {
        if (NT == 64) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    static __device__ Seen join(Seen v, float c, Shared &s)
    {
        v = wave_join(v, c);
        if (NT == 64) return v;
        if ((threadIdx.x & 63) == 0) {
            const int w = threadIdx.x >> 6;
            s.top[w] = v.top;
            s.sum[w] = v.sum;
            s.sum2[w] = v.sum2;
        }
        sync();
        Seen all;
        for (int w = 0; w < kWaves; ++w) all.top = fmaxf(all.top, s.top[w]);
        for (int w = 0; w < kWaves; ++w) {
            Seen one;
            one.top = s.top[w];
            one.sum = s.sum[w];
            one.sum2 = s.sum2[w];
            one.raise(all.top, c);
            all.sum += one.sum;
            all.sum2 += one.sum2;
        }
        return all;
    }
    // sum over the team of a count that is the same in all lanes of a wave; `turn` alternates from call to call
    static __device__ uint32_t count(uint32_t n, int turn, Shared &s)
    {
        if (NT == 64) return n;
        if ((threadIdx.x & 63) == 0) s.count[turn & 1][threadIdx.x >> 6] = n;
        sync();
        uint32_t all = 0;
        for (int w = 0; w < kWaves; ++w) all += s.count[turn & 1][w];
        return all;
    }
    static __device__ uint64_t max_place(uint64_t x, uint64_t *slots)
    {
        x = wave_reduce(x, (uint64_t)0, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        if (NT == 64) return x;
        sync();
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
        sync();
        for (int w = 0; w < kWaves; ++w) x = slots[w] > x ? slots[w] : x;
        return x;
    }
    // A place that at least `least` of the places, one a thread, are at or above: the lowest of what every wave finds by taking off its largest so many times.
    // 0 where a wave has fewer.
    static __device__ uint64_t low_threshold(uint32_t least, uint64_t x, uint64_t *slots)
    {
        uint64_t last = 0;
        for (uint32_t i = 0; i < (least + kWaves - 1) / kWaves; ++i) {
            last = wave_reduce(x, (uint64_t)0, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
            if (x == last) x = 0;
        }
        if (NT == 64) return last;
        sync();
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = last;
        sync();
        for (int w = 0; w < kWaves; ++w) last = slots[w] < last ? slots[w] : last;
        return last;
    }
    // A place that at least `least` and at most `most` of the places are at or above, of which at_or_above(p) counts the wave's; 1 if there are
    // fewer than `least`.  hi: an upper bound of all places.  The range is halved, 64 times at most.
    template <typename F>
    static __device__ uint64_t threshold(uint32_t least, uint32_t most, uint64_t hi, F at_or_above, Shared &s)
    {
        uint64_t lo = 1;                                 // at or above lo: at least `least`, or too few altogether; above hi: none
        int turn = 0;
        if (count(at_or_above(lo), turn++, s) < least) {
            if (NT != 64) sync();
            return lo;
        }
        // (logits that lead lie close to each other: the first steps look down from the largest, each twice as far)
        for (uint64_t step = 1ull << 52; hi > lo && step < hi - lo; step <<= 1) {
            const uint64_t at = hi - step;
            const uint32_t n = count(at_or_above(at), turn++, s);
            if (n >= least) {
                lo = at;
                if (n <= most) hi = at;
                break;
            }
            hi = at - 1;
        }
        while (lo < hi) {
            const uint64_t at = lo + (hi - lo + 1) / 2;
            const uint32_t n = count(at_or_above(at), turn++, s);
            if (n >= least) {
                lo = at;
                if (n <= most) break;
            } else {
                hi = at - 1;
            }
        }
        if (NT != 64) sync();
        return lo;
    }
};
__device__ inline uint32_t wave_count(bool x) { return (uint32_t)__popcll(__ballot(x)); }

// The entries [begin, end) of a row, packs one thread after the other, so many read ahead; f(index, pack) for whole packs, g(index, x) for what is left
template <typename T, int NT, int AHEAD, typename F, typename G>
__device__ inline void for_entries(const T *x, int64_t begin, int64_t end, F f, G g)
{
    constexpr int N = Pack<T>::N;
    const int t = Team<NT>::tid();
    const int64_t packs = (end - begin) / N, rest = begin + packs * N;
    const T *const p = x + begin;
    int64_t i = t;
    if (AHEAD > 1) {
        for (; i + (AHEAD - 1) * NT < packs; i += AHEAD * NT) {
            Pack<T> v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) v[j] = load_pack(p + (i + j * NT) * N);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) f(begin + (i + j * NT) * N, v[j]);
        }
    }
#pragma unroll 1
    for (; i < packs; i += NT) f(begin + i * N, load_pack(p + i * N));
    for (int64_t j = rest + t; j < end; j += NT) g(j, x[j]);
}

// One pass over entries [begin, end): what has been seen, and (with TOP) the thread's best place
template <typename T, int NT, bool TOP>
__device__ inline Seen read_row(const T *x, int64_t begin, int64_t end, float c, uint64_t *best)
{
    Seen s;
    uint64_t b = 0;
    const auto one = [&](int64_t j, T raw) {
        const float v = logit_of(raw);
        if (v > s.top) {
            s.raise(v, c);
            if (TOP) b = place_of(v, (uint32_t)j);
        }
        s.add(v, c);
    };
    for_entries<T, NT, 4>(x, begin, end, [&](int64_t j, const Pack<T> &p) {
        constexpr int N = Pack<T>::N;
        float v[N], top = s.top;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = logit_of(p.x[i]), top = fmaxf(top, v[i]);
        if (top > s.top) {
            s.raise(top, c);
            if (TOP) {
                int at = N - 1;
#pragma unroll
                for (int i = N - 2; i >= 0; --i) at = v[i] == top ? i : at;
                b = place_of(top, (uint32_t)(j + at));
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) s.add(v[i], c);
    }, one);
    if (TOP) *best = b;
    return s;
}

// The `top` best of the places that the list holds (there may be fewer), in order: put(rank, place), for the ranks that there are
template <int NT, typename F>
__device__ inline void best_of_list(uint64_t *list, uint64_t *few, uint32_t n, uint32_t top, typename Team<NT>::Shared &s, uint64_t *slots, F put)
{
    using Tm = Team<NT>;
    const int t = Tm::tid();
    const uint64_t *from = list;
    if (n > kRanked) {
        uint64_t mine = 0;
        for (uint32_t i = t; i < n; i += NT) mine = list[i] > mine ? list[i] : mine;
        const uint64_t hi = Tm::max_place(mine, slots);
        const uint64_t least = Tm::threshold(top, kRanked, hi, [&](uint64_t p) {
            uint32_t c = 0;
            for (uint32_t i = t; i < (n + NT - 1) / NT * NT; i += NT) c += wave_count(i < n && list[i] >= p);
            return c;
        }, s);
        if (t == 0) s.listed = 0;
        Tm::sync();
        for (uint32_t i = t; i < n; i += NT)
            if (list[i] >= least) {
                const uint32_t at = atomicAdd(&s.listed, 1u);
                if (at < kRanked) few[at] = list[i];
            }
        Tm::sync();
        n = s.listed < (uint32_t)kRanked ? s.listed : (uint32_t)kRanked;
        from = few;
    }
    // so many lanes count what is before an entry
    const uint32_t lanes = n * 8 <= NT ? 8 : n * 4 <= NT ? 4 : n * 2 <= NT ? 2 : 1;
    for (uint32_t first = 0; first < n; first += NT / lanes) {
        const uint32_t i = first + t / lanes;
        const uint64_t mine = i < n ? from[i] : 0;
        uint32_t before = 0;
#pragma unroll 4
        for (uint32_t j = t & (lanes - 1); j < n; j += lanes) before += from[j] > mine;
        for (uint32_t d = 1; d < lanes; d <<= 1) before += __shfl_xor(before, d);
        if (i < n && (t & (lanes - 1)) == 0 && before < top) put(before, mine);
    }
}

// The `top` best of entries [begin, end) that the team has just read, a thread's best place being `best`
template <typename T, int NT, typename F>
__device__ inline void best_of_row(const T *x, int64_t begin, int64_t end, uint32_t top, uint64_t best, uint64_t *list, uint64_t *few,
                                   typename Team<NT>::Shared &s, uint64_t *slots, F put)
{
    using Tm = Team<NT>;
    const auto list_from = [&](uint64_t least, bool mine) {
        Tm::sync();
        if (Tm::tid() == 0) s.listed = 0;
        Tm::sync();
        const auto one = [&](int64_t j, T raw) {
            const uint64_t p = place_of(logit_of(raw), (uint32_t)j);
            if (p >= least) {
                const uint32_t at = atomicAdd(&s.listed, 1u);
                if (at < (uint32_t)kListed) list[at] = p;
            }
        };
        if (mine)
            for_entries<T, NT, 1>(x, begin, end, [&](int64_t j, const Pack<T> &p) {
                float most = -INFINITY;
#pragma unroll
                for (int i = 0; i < Pack<T>::N; ++i) most = fmaxf(most, logit_of(p.x[i]));
                if (most < logit_at(least)) return;      // (a threshold below every number's is none)
                uint32_t found = 0;
#pragma unroll
                for (int i = 0; i < Pack<T>::N; ++i) found += place_of(logit_of(p.x[i]), (uint32_t)(j + i)) >= least;
                if (found == 0) return;
                uint32_t at = atomicAdd(&s.listed, found);
#pragma unroll
                for (int i = 0; i < Pack<T>::N; ++i) {
                    const uint64_t place = place_of(logit_of(p.x[i]), (uint32_t)(j + i));
                    if (place >= least && at < (uint32_t)kListed) list[at] = place;
                    at += place >= least;
                }
            }, one);
        Tm::sync();
        return s.listed;
    };
    uint64_t least = 1, hi = 0;
    if (NT > 64) {                                       // (a wave lists its whole row)
        // (a few rounds in every wave and one barrier; halving the range of places takes some 20 of both)
        least = top <= 8 * Tm::kWaves ? Tm::low_threshold(top, best, slots) : 0;
        if (least == 0) {
            hi = Tm::max_place(best, slots);
            least = Tm::threshold(top, 2 * top, hi, [&](uint64_t p) { return wave_count(best >= p); }, s);
        }
    }
    uint32_t n;
#pragma unroll 1
    for (bool mine = best >= least;; mine = true) {
        n = list_from(least, mine);
        if (n <= (uint32_t)kListed) break;
        // many large logits with few threads: the row is counted again and again, until the list holds them
        if (hi == 0) hi = Tm::max_place(best, slots);
        least = Tm::threshold(top, kListed, hi, [&](uint64_t p) {
            uint32_t c = 0;
            for_entries<T, NT, 1>(x, begin, end, [&](int64_t j, const Pack<T> &v) {
#pragma unroll 1
                for (int i = 0; i < Pack<T>::N; ++i) c += place_of(logit_of(v.x[i]), (uint32_t)(j + i)) >= p;
            }, [&](int64_t j, T raw) { c += place_of(logit_of(raw), (uint32_t)j) >= p; });
            return (uint32_t)wave_sum((uint64_t)c);
        }, s);
    }
    best_of_list<NT>(list, few, n, top, s, slots, put);
}

// Fills the ranks from `n` on
template <int NT>
__device__ inline void no_alternatives(const RowArgs &a, int64_t row, uint32_t n)
{
    for (uint32_t i = n + Team<NT>::tid(); i < (uint32_t)a.top; i += NT) {
        a.top_logprob[row * a.top + i] = -INFINITY;
        a.top_token[row * a.top + i] = -1;
    }
}
__device__ inline void put_alternative(const RowArgs &a, int64_t row, const Seen &v, float inv, float log, uint32_t rank, uint64_t place)
{
    a.top_logprob[row * a.top + rank] = v.logprob(logit_at(place), inv, log);
    a.top_token[row * a.top + rank] = (int32_t)index_at(place);
}

template <typename T>
__device__ inline void put_row(const RowArgs &a, int64_t row, const T *x, const Seen &v, float inv, float log)
{
    if (a.entropy) a.entropy[row] = v.entropy();
    if (a.norm) a.norm[2 * row] = v.top, a.norm[2 * row + 1] = log;
    if (a.logprob) {
        const int32_t token = a.token[row];
        a.logprob[row] = token >= 0 && token < a.n ? v.logprob(logit_of(x[token]), inv, log) : 0.0f;
    }
}

__device__ inline float teacher_at(const RowArgs &a, int64_t i)
{
    const float x = a.teacher_type == RLS_F32 ? static_cast<const float *>(a.teacher)[i]
                    : a.teacher_type == RLS_BF16 ? (float)static_cast<const __bf16 *>(a.teacher)[i] : (float)static_cast<const _Float16 *>(a.teacher)[i];
    return x > kLargest ? kLargest : x;
}
// What the lanes that take a row have of its teacher: 128 entries among them; entries that do not count are at -infinity
template <int L>
struct Teacher {
    static constexpr int E = RLS_MAX_TOP / L;
    float x[E];
    int32_t token[E];
    float top, sum;

    __device__ void load(const RowArgs &a, int64_t row, float c)
    {
        const int lane = threadIdx.x & (L - 1);
        top = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = -INFINITY;
            token[e] = -1;
            const int j = lane + L * e;
            if (L * e < a.k && j < a.k) {
                token[e] = a.token[row * a.k + j];
                const float v = teacher_at(a, row * a.k + j);
                if (token[e] >= 0 && token[e] < a.n && v > -INFINITY) x[e] = v;
            }
            top = fmaxf(top, x[e]);
        }
        top = lanes_max<L>(top);
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += power_of(distance2(x[e], top, c));
        sum = lanes_sum<L>(sum);
    }
    __device__ float share(int e, float c) const { return sum > 0.0f ? power_of(distance2(x[e], top, c)) / sum : 0.0f; }
};
// The loss of a row
template <int L, typename T>
__device__ inline void put_loss(const RowArgs &a, int64_t row, bool live, const T *x, const Seen &v, float inv, float log, const Teacher<L> &t)
{
    const float log_teacher = t.sum > 0.0f ? logf(t.sum) : 0.0f;
    float loss = 0.0f;
#pragma unroll
    for (int e = 0; e < Teacher<L>::E; ++e) {
        const float p = t.share(e, inv * kLog2e);
        if (p > 0.0f) loss = fmaf(p, ((t.x[e] - t.top) * inv - log_teacher) - v.logprob(logit_of(x[t.token[e]]), inv, log), loss);
    }
    loss = lanes_sum<L>(loss);
    if ((threadIdx.x & (L - 1)) == 0 && live) {
        a.logprob[row] = loss;
        if (a.norm) a.norm[2 * row] = v.top, a.norm[2 * row + 1] = log;
    }
}

// ---- rows that a thread takes ----------------------------------------------------------------------------------------

template <typename T, int N>
__global__ void __launch_bounds__(256) logprobs_thread_kernel(RowArgs a)
{
    const int64_t row = a.row0 + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const int n = (int)a.n;
    const float inv = inverse_of(a.temperature, row), c = inv * kLog2e;
    float l[N];
    Seen v;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        l[i] = i < n ? logit_of(x[i]) : -INFINITY;
        v.top = fmaxf(v.top, l[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v.add(l[i], c);
    const float log = v.log_sum();
    put_row(a, row, x, v, inv, log);
    if (a.top == 0) return;
    uint32_t live = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!(l[i] > -INFINITY)) continue;
        ++live;
        uint32_t before = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) before += j < i ? l[j] >= l[i] : l[j] > l[i];
        if (before < (uint32_t)a.top) put_alternative(a, row, v, inv, log, before, place_of(l[i], (uint32_t)i));
    }
    for (uint32_t i = live; i < (uint32_t)a.top; ++i) {
        a.top_logprob[row * a.top + i] = -INFINITY;
        a.top_token[row * a.top + i] = -1;
    }
}

// ---- rows that 16 lanes take, or a wave, in registers: P packs a lane ---------------------------------------------------
// Alternatives are taken off one after the other: the best of the lanes' best places, whose lane then looks for its next.

constexpr int kTakenOff = 16;                            // alternatives; more go through a list

template <typename T, int L, int P, bool TOP, bool TEACHER>
__global__ void __launch_bounds__(256) logprobs_lanes_kernel(RowArgs a)
{
    constexpr int N = Pack<T>::N;
    const int lane = threadIdx.x & (L - 1), n = (int)a.n;
    const int64_t at = a.row0 + (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L, row = min(at, a.rows - 1);
    const bool live = at < a.rows;                       // (the others go along with the last row)
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const float inv = inverse_of(a.temperature, row), c = inv * kLog2e;
    Teacher<L> teacher;
    if (TEACHER) teacher.load(a, row, c);
    float v[P][N];
    Seen s;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int first = (i * L + lane) * N;
        if (first + N <= n) {
            const Pack<T> raw = load_pack(x + first);
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = logit_of(raw.x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = first + e < n ? logit_of(x[first + e]) : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) s.top = fmaxf(s.top, v[i][e]);
    }
    s.top = lanes_max<L>(s.top);
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) s.add(v[i][e], c);
    s.sum = lanes_sum<L>(s.sum);
    s.sum2 = lanes_sum<L>(s.sum2);
    const float log = s.log_sum();
    if (TEACHER) {
        put_loss<L>(a, row, live, x, s, inv, log, teacher);
        return;
    }
    if (lane == 0 && live) put_row(a, row, x, s, inv, log);
    if (!TOP) return;
    const auto best_below = [&](uint64_t limit) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint64_t place = place_of(v[i][e], (uint32_t)((i * L + lane) * N + e));
                if (place < limit && place > best) best = place;
            }
        return best;
    };
    uint64_t mine = best_below(~0ull);
#pragma unroll 1
    for (int rank = 0; rank < a.top; ++rank) {
        const uint64_t best = lanes_reduce<L>(mine, (uint64_t)0, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
        if (best == 0 ? lane == 0 : mine == best) {
            if (live) {
                a.top_logprob[row * a.top + rank] = best == 0 ? -INFINITY : s.logprob(logit_at(best), inv, log);
                a.top_token[row * a.top + rank] = best == 0 ? -1 : (int32_t)index_at(best);
            }
            mine = best_below(best);
        }
    }
}

// ---- rows that a wave or a workgroup takes ---------------------------------------------------------------------------

template <int NT, bool TOP>
struct RowShared {
    typename Team<NT>::Shared team;
    uint64_t slots[NT / 64];
    uint64_t list[TOP ? (NT == 64 ? kWaveRow : kListed) : 1], few[TOP ? kRanked : 1];
};

template <typename T, int NT, bool TOP, bool TEACHER>
__global__ void __launch_bounds__(NT == 64 ? 256 : NT) logprobs_row_kernel(RowArgs a)
{
    using Tm = Team<NT>;
    __shared__ RowShared<NT, TOP> shared[NT == 64 ? 4 : 1];
    RowShared<NT, TOP> &s = shared[NT == 64 ? threadIdx.x >> 6 : 0];
    const int64_t row = a.row0 + (NT == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x);
    if (row >= a.rows) return;                           // (whole waves, whole workgroups)
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const float inv = inverse_of(a.temperature, row), c = inv * kLog2e;
    Teacher<64> teacher;
    if (TEACHER && (NT == 64 || threadIdx.x < 64)) teacher.load(a, row, c);
    uint64_t best = 0;
    const Seen v = Tm::join(read_row<T, NT, TOP>(x, 0, a.n, c, &best), c, s.team);
    const float log = v.log_sum();
    if (TEACHER) {
        if (NT == 64 || threadIdx.x < 64) put_loss<64>(a, row, true, x, v, inv, log, teacher);
        return;
    }
    if (Tm::tid() == 0) put_row(a, row, x, v, inv, log);
    if (TOP) {
        no_alternatives<NT>(a, row, 0);
        Tm::sync();
        best_of_row<T, NT>(x, 0, a.n, (uint32_t)a.top, best, s.list, s.few, s.team, s.slots,
                           [&](uint32_t rank, uint64_t place) { put_alternative(a, row, v, inv, log, rank, place); });
    }
}

// ---- rows in pieces, a workgroup each, joined by another launch ------------------------------------------------------

constexpr int kPieceThreads = 512;

template <typename T, bool TOP>
__global__ void __launch_bounds__(kPieceThreads) logprobs_piece_kernel(RowArgs a)
{
    using Tm = Team<kPieceThreads>;
    __shared__ RowShared<kPieceThreads, TOP> s;
    const int64_t row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const int64_t begin = piece * a.piece, end = min(a.n, begin + a.piece);
    const float c = inverse_of(a.temperature, row) * kLog2e;
    uint64_t best = 0;
    const Seen v = Tm::join(read_row<T, kPieceThreads, TOP>(x, begin, end, c, &best), c, s.team);
    if (threadIdx.x == 0) {
        float *const part = a.part + (row * a.pieces + piece) * 4;
        part[0] = v.top;
        part[1] = v.sum;
        part[2] = v.sum2;
    }
    if (TOP) {
        uint64_t *const out = a.best + (row * a.pieces + piece) * a.top;
        for (int i = threadIdx.x; i < a.top; i += kPieceThreads) out[i] = 0;
        __syncthreads();
        best_of_row<T, kPieceThreads>(x, begin, end, (uint32_t)a.top, best, s.list, s.few, s.team, s.slots,
                                      [&](uint32_t rank, uint64_t place) { out[rank] = place; });
    }
}

constexpr int kJoinThreads = 1024;

template <typename T, bool TOP, bool TEACHER>
__global__ void __launch_bounds__(kJoinThreads) logprobs_join_kernel(RowArgs a)
{
    using Tm = Team<kJoinThreads>;
    __shared__ RowShared<kJoinThreads, TOP> s;
    const int64_t row = blockIdx.x;
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    const float inv = inverse_of(a.temperature, row), c = inv * kLog2e;
    Teacher<64> teacher;
    if (TEACHER && threadIdx.x < 64) teacher.load(a, row, c);
    Seen mine;
    for (int i = threadIdx.x; i < a.pieces; i += kJoinThreads) {
        const float *const part = a.part + (row * a.pieces + i) * 4;
        Seen one;
        one.top = part[0];
        one.sum = part[1];
        one.sum2 = part[2];
        const float top = fmaxf(one.top, mine.top);
        mine.raise(top, c);
        one.raise(top, c);
        mine.sum += one.sum;
        mine.sum2 += one.sum2;
    }
    const Seen v = Tm::join(mine, c, s.team);
    const float log = v.log_sum();
    if (TEACHER) {
        if (threadIdx.x < 64) put_loss<64>(a, row, true, x, v, inv, log, teacher);
        return;
    }
    if (threadIdx.x == 0) put_row(a, row, x, v, inv, log);
    if (TOP) {
        if (threadIdx.x == 0) s.team.listed = 0;
        no_alternatives<kJoinThreads>(a, row, 0);
        __syncthreads();
        const int n = a.pieces * a.top;                  // (at most kListed)
        for (int i = threadIdx.x; i < n; i += kJoinThreads) {
            const uint64_t p = a.best[row * n + i];
            if (p != 0) s.list[atomicAdd(&s.team.listed, 1u)] = p;
        }
        __syncthreads();
        const uint32_t listed = s.team.listed;
        __syncthreads();
        best_of_list<kJoinThreads>(s.list, s.few, listed, (uint32_t)a.top, s.team, s.slots,
                                   [&](uint32_t rank, uint64_t place) { put_alternative(a, row, v, inv, log, rank, place); });
    }
}

// ---- gradients ---------------------------------------------------------------------------------------------------------

struct GradArgs {
    RowArgs row;                                         // norm and entropy are read
    const float *by_logprob, *by_entropy;                // distill: by_logprob is the gradient by the loss
    void *out;
    int64_t ld_out, piece;
    int32_t pieces;
};

// dx = inv ((token's entry: at_token) - p (each + by_log log p)).  inv comes last: what it is multiplied with may be the small difference of large numbers, and
// 0 where inv is as large as it gets
struct Slope {
    float top, c, inv, log2_sum, at_token, each, by_log;
    int32_t token;
};
__device__ inline Slope slope_of(const GradArgs &g, int64_t row)
{
    const RowArgs &a = g.row;
    const float inv = inverse_of(a.temperature, row);
    Slope s;
    s.top = a.norm[2 * row];
    s.c = inv * kLog2e;
    s.inv = inv;
    s.log2_sum = a.norm[2 * row + 1] * kLog2e;
    s.token = a.token ? a.token[row] : -1;
    const bool given = s.token >= 0 && s.token < a.n && g.by_logprob;
    s.at_token = given ? g.by_logprob[row] : 0.0f;
    s.by_log = g.by_entropy ? g.by_entropy[row] : 0.0f;
    s.each = s.at_token + (g.by_entropy ? s.by_log * a.entropy[row] : 0.0f);
    if (!given) s.token = -1;
    return s;
}
// without inv (an entry whose probability is 0 has no part in the entropy, and its gradient is 0 whatever the factors are)
__device__ inline float slope_at(const Slope &s, float x)
{
    const float l2 = distance2(x, s.top, s.c) - s.log2_sum, p = power_of(l2);
    return p > 0.0f ? -p * fmaf(s.by_log, l2 * kLn2, s.each) : 0.0f;
}
template <typename T>
__device__ inline float slope_at_token(const Slope &s, T raw, float d)
{
    const float x = logit_of(raw);
    return x > -INFINITY ? d + s.at_token : 0.0f;
}

template <typename T, int N>
__global__ void __launch_bounds__(256) logprobs_grad_thread_kernel(GradArgs g)
{
    const int64_t row = g.row.row0 + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= g.row.rows) return;
    const T *const x = static_cast<const T *>(g.row.logits) + row * g.row.ld;
    T *const out = static_cast<T *>(g.out) + row * g.ld_out;
    const int n = (int)g.row.n;
    const Slope s = slope_of(g, row);
    T l[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) l[i] = x[i];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i >= n) continue;
        float d = slope_at(s, logit_of(l[i]));
        if (i == s.token) d = slope_at_token(s, l[i], d);
        out[i] = (T)(d * s.inv);
    }
}

// A piece of a row by a workgroup (L = 256), or a whole row by 16 lanes or a wave; TEACHER: the teacher's entries are written after the others
template <typename T, int L, bool TEACHER>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(GradArgs g)
{
    constexpr int N = Pack<T>::N, R = 256 / L, W = L < 64 ? L : 64, E = RLS_MAX_TOP / W;
    __shared__ float share[TEACHER ? R : 1][RLS_MAX_TOP];
    __shared__ int32_t where[TEACHER ? R : 1][RLS_MAX_TOP];
    __shared__ bool taught[R];
    const auto sync = [] {
        if (L == 256) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    const RowArgs &a = g.row;
    const int lane = threadIdx.x & (L - 1), team = L == 256 ? 0 : threadIdx.x / L;      // (a workgroup's row is known to be one)
    const int64_t unit = (int64_t)blockIdx.x * R + team, at = a.row0 + unit / g.pieces, row = min(at, a.rows - 1);
    const int64_t begin = unit % g.pieces * g.piece, end = at < a.rows ? min(a.n, begin + g.piece) : begin;        // (nothing of the rows behind the last)
    const T *const x = static_cast<const T *>(a.logits) + row * a.ld;
    T *const out = static_cast<T *>(g.out) + row * g.ld_out;
    Slope s;
    float late[E];                                       // what entries of the teacher that lie in this piece get
    int32_t late_at[E];
    if (TEACHER) {
        const float inv = inverse_of(a.temperature, row);
#pragma unroll
        for (int e = 0; e < E; ++e) late_at[e] = -1;
        Teacher<W> t;
        if (lane < W) {
            t.load(a, row, inv * kLog2e);
            if (lane == 0) taught[team] = t.sum > 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float p = t.share(e, inv * kLog2e);
                share[team][lane + W * e] = p;
                where[team][lane + W * e] = p > 0.0f ? t.token[e] : -1;
            }
        }
        sync();
        s.top = a.norm[2 * row];
        s.c = inv * kLog2e;
        s.inv = inv;
        s.log2_sum = a.norm[2 * row + 1] * kLog2e;
        s.by_log = 0.0f;
        s.token = -1;
        s.at_token = taught[team] ? -g.by_logprob[row] : 0.0f;
        s.each = s.at_token;
        // an entry of the teacher: its first place in the list writes it, with what all its places have
        if (lane < W) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int mine = lane + W * e;
                const int32_t to = where[team][mine];
                if (W * e >= a.k || to < begin || to >= end) continue;
                float p = 0.0f;
                bool first = true;
                for (int j = 0; j < a.k; ++j) {
                    const bool same = where[team][j] == to;
                    if (same && j < mine) first = false;
                    p += same ? share[team][j] : 0.0f;
                }
                const float v = logit_of(x[to]);
                if (first && v > -INFINITY) {
                    const float l2 = distance2(v, s.top, s.c) - s.log2_sum;
                    late[e] = -s.each * (power_of(l2) - p) * s.inv;
                    late_at[e] = to;
                }
            }
        }
        sync();                                          // the logits may lie where the gradients go
    } else {
        s = slope_of(g, row);
    }
    const auto pack = [&](int64_t j, const Pack<T> &p) {
        Pack<T> d;
#pragma unroll
        for (int i = 0; i < N; ++i) d.x[i] = (T)(slope_at(s, logit_of(p.x[i])) * s.inv);
        if (!TEACHER && s.token >= j && s.token < j + N) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (s.token == j + i) d.x[i] = (T)(slope_at_token(s, p.x[i], slope_at(s, logit_of(p.x[i]))) * s.inv);
        }
        store_pack(out + j, d);
    };
    const auto one = [&](int64_t j, T raw) {
        float d = slope_at(s, logit_of(raw));
        if (!TEACHER && s.token == j) d = slope_at_token(s, raw, d);
        out[j] = (T)(d * s.inv);
    };
    const int64_t packs = (end - begin) / N;
    if (L == 256) {
        int64_t i = lane;
        for (; i + 3 * L < packs; i += 4 * L) {
            Pack<T> v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = load_pack(x + begin + (i + j * L) * N);
#pragma unroll
            for (int j = 0; j < 4; ++j) pack(begin + (i + j * L) * N, v[j]);
        }
#pragma unroll 1
        for (; i < packs; i += L) pack(begin + i * N, load_pack(x + begin + i * N));
    } else {
#pragma unroll 1
        for (int i = lane; i < packs; i += L) pack(begin + i * N, load_pack(x + begin + i * N));
    }
    for (int64_t j = begin + packs * N + lane; j < end; j += L) one(j, x[j]);
    if (TEACHER) {
        sync();                                          // (what was stored before the barrier comes before what is stored behind it)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (late_at[e] >= 0) out[late_at[e]] = (T)late[e];
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------

// A row is cut where there are too few rows to fill the card: into pieces of at least 8192 entries, 1024 of them in all
struct Cut {
    int64_t piece;
    int32_t pieces;
    int64_t best, total;                                 // of the workspace: where the best places begin, and its size
};
Cut cut_of(int64_t rows, int64_t n, int32_t top)
{
    Cut c{n, 1, 0, 0};
    if (n <= 16384 || rows >= 512) return c;
    int64_t pieces = std::min<int64_t>((1024 + rows - 1) / rows, n / 8192);
    if (top > 0) pieces = std::min<int64_t>(pieces, std::max<int64_t>(4, kRanked / top));         // (the join counts their lists at once)
    if (pieces <= 1) return c;
    c.piece = align_up((n + pieces - 1) / pieces, 64);
    c.pieces = (int32_t)((n + c.piece - 1) / c.piece);
    c.best = align_up(rows * c.pieces * 16, 256);
    c.total = c.best + align_up(rows * c.pieces * (int64_t)top * 8, 256);
    return c;
}

// every row by a workgroup of one size: rows of many entries by 256 threads where there are enough of them to fill the card, else by 1024
int threads_of(int64_t rows, int64_t n)
{
    if (n <= kWaveRow) return 64;
    return n <= 8192 || rows >= 1024 ? 256 : 1024;
}

// A launch has less than 2^32 threads: rows [first, first + most) by each
template <typename F>
hipError_t by_rows(RowArgs &a, int64_t most, F launch)
{
    const int64_t rows = a.rows;
    for (a.row0 = 0; a.row0 < rows; a.row0 += most) {
        a.rows = std::min(rows, a.row0 + most);
        launch(a.rows - a.row0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
constexpr int64_t kMostRows = 1 << 21;

template <typename T, int NT>
hipError_t launch_rows(RowArgs a, hipStream_t s)
{
    void (*kernel)(RowArgs) = logprobs_row_kernel<T, NT, true, false>;
    if constexpr (NT > 64) {                             // (rows of a wave come here for their alternatives only)
        if (a.top == 0) kernel = a.teacher ? logprobs_row_kernel<T, NT, false, true> : logprobs_row_kernel<T, NT, false, false>;
    }
    return by_rows(a, kMostRows, [&](int64_t rows) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(NT == 64 ? (rows + 3) / 4 : rows)), dim3(NT == 64 ? 256 : NT), 0, s, a);
    });
}

template <typename T, int L, int P>
hipError_t launch_lanes(RowArgs a, hipStream_t s)
{
    auto *const kernel = a.teacher ? logprobs_lanes_kernel<T, L, P, false, true>
                         : a.top > 0 ? logprobs_lanes_kernel<T, L, P, true, false> : logprobs_lanes_kernel<T, L, P, false, false>;
    return by_rows(a, kMostRows, [&](int64_t rows) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 256 / L - 1) / (256 / L))), dim3(256), 0, s, a);
    });
}

template <typename T>
hipError_t launch_forward(RowArgs a, char *ws, hipStream_t s)
{
    if (!a.teacher && a.n <= kThreadRow) {
        auto *const kernel = a.n <= 4 ? logprobs_thread_kernel<T, 4> : a.n <= 8 ? logprobs_thread_kernel<T, 8> : logprobs_thread_kernel<T, 16>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    // 16 lanes for rows of up to 256 entries (524288 x 20 in fp32 with a wave a row: 128 us, with 3 alternatives 602)
    if (a.n <= kWaveRow && a.top <= kTakenOff) {
        constexpr int N = Pack<T>::N;
        if (a.n <= 16 * N) return launch_lanes<T, 16, 1>(a, s);
        if (a.n <= 256) return launch_lanes<T, 16, 256 / (16 * N)>(a, s);
        if (a.n <= 64 * N) return launch_lanes<T, 64, 1>(a, s);
        return launch_lanes<T, 64, kWaveRow / (64 * N)>(a, s);
    }
    const Cut c = cut_of(a.rows, a.n, a.top);
    if (c.pieces == 1) {
        const int threads = threads_of(a.rows, a.n);
        return threads == 64 ? launch_rows<T, 64>(a, s) : threads == 256 ? launch_rows<T, 256>(a, s) : launch_rows<T, 1024>(a, s);
    }
    a.pieces = c.pieces;
    a.piece = c.piece;
    a.part = reinterpret_cast<float *>(ws);
    a.best = reinterpret_cast<uint64_t *>(ws + c.best);
    auto *const piece = a.top > 0 ? logprobs_piece_kernel<T, true> : logprobs_piece_kernel<T, false>;
    hipLaunchKernelGGL(piece, dim3((unsigned)(a.rows * c.pieces)), dim3(kPieceThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto *const join = a.teacher ? logprobs_join_kernel<T, false, true> : a.top > 0 ? logprobs_join_kernel<T, true, false> : logprobs_join_kernel<T, false, false>;
    hipLaunchKernelGGL(join, dim3((unsigned)a.rows), dim3(kJoinThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_backward(GradArgs g, hipStream_t s)
{
    RowArgs &a = g.row;
    if (!a.teacher && a.n <= kThreadRow) {
        auto *const kernel = a.n <= 4 ? logprobs_grad_thread_kernel<T, 4> : a.n <= 8 ? logprobs_grad_thread_kernel<T, 8> : logprobs_grad_thread_kernel<T, 16>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, g);
        return hipGetLastError();
    }
    if (a.n <= kWaveRow) {                               // 16 lanes a row up to 256 entries, else a wave (524288 x 20 in bf16 with a wave a row: 448 us)
        const int lanes = a.n <= 256 ? 16 : 64;
        g.piece = kWaveRow;
        g.pieces = 1;
        auto *const kernel = lanes == 16 ? (a.teacher ? logprobs_grad_kernel<T, 16, true> : logprobs_grad_kernel<T, 16, false>)
                             : (a.teacher ? logprobs_grad_kernel<T, 64, true> : logprobs_grad_kernel<T, 64, false>);
        return by_rows(a, kMostRows, [&](int64_t rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 256 / lanes - 1) / (256 / lanes))), dim3(256), 0, s, g);
        });
    }
    // pieces of at most 8192 entries; of fewer, down to 2048, where there are few rows (8192 x 32001 in bf16: 218 us with 16384, 211 with 8192)
    g.piece = std::min<int64_t>(8192, std::max<int64_t>(2048, align_up((a.rows * a.n + 2047) / 2048, 64)));
    g.pieces = (int32_t)((a.n + g.piece - 1) / g.piece);
    auto *const kernel = a.teacher ? logprobs_grad_kernel<T, 256, true> : logprobs_grad_kernel<T, 256, false>;
    return by_rows(a, std::max<int64_t>(1, (1 << 23) / g.pieces), [&](int64_t rows) { hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * g.pieces)), dim3(256), 0, s, g); });
}

int32_t check_rows(const void *logits, int32_t type, int64_t rows, int64_t n, int64_t ld)
{
    if (!logits) return RLS_ERR_NULL;
    if (rows < 1 || rows > RLS_MAX_N || n < 1 || n > RLS_MAX_CHOICES || !is_type(type)) return RLS_ERR_INVALID_ARG;
    return ld < n || ld > (1LL << 40) / rows ? RLS_ERR_SHAPE : RLS_OK;      // (no memory reaches that far)
}

// bytes from..to of an array
struct Span {
    uintptr_t from = 0, to = 0;
    Span() = default;
    Span(const void *p, int64_t bytes) : from((uintptr_t)p), to(p ? from + (uintptr_t)bytes : from) {}
    bool meets(const Span &o) const { return from < o.to && o.from < to; }
};
Span matrix(const void *p, int64_t rows, int64_t n, int64_t ld, int64_t element) { return {p, ((rows - 1) * ld + n) * element}; }
int32_t check_apart(std::initializer_list<Span> written, std::initializer_list<Span> read)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (const Span &r : read)
            if (w->meets(r)) return RLS_ERR_SHAPE;
        for (auto v = written.begin(); v != w; ++v)
            if (w->meets(*v)) return RLS_ERR_SHAPE;
    }
    return RLS_OK;
}

int32_t check_space(int64_t need, const void *ws, int64_t bytes)
{
    return need > 0 && (!ws || (uintptr_t)ws % 256 != 0 || bytes < need) ? RLS_ERR_WORKSPACE : RLS_OK;
}
template <typename F32, typename B16, typename H16>
hipError_t by_type(int32_t type, F32 f, B16 b, H16 h)
{
    return type == RLS_F32 ? f() : type == RLS_BF16 ? b() : h();
}
hipError_t forward(int32_t type, const RowArgs &a, char *ws, hipStream_t s)
{
    return by_type(type, [&] { return launch_forward<float>(a, ws, s); }, [&] { return launch_forward<__bf16>(a, ws, s); },
                   [&] { return launch_forward<_Float16>(a, ws, s); });
}
hipError_t backward(int32_t type, const GradArgs &g, hipStream_t s)
{
    return by_type(type, [&] { return launch_backward<float>(g, s); }, [&] { return launch_backward<__bf16>(g, s); },
                   [&] { return launch_backward<_Float16>(g, s); });
}
// the gradients go where the logits are, entry by entry, or where nothing else is
int32_t check_gradients(const RowArgs &a, int64_t element, const void *out, int64_t ld_out, std::initializer_list<Span> read)
{
    if (!out) return RLS_ERR_NULL;
    if (ld_out < a.n || ld_out > (1LL << 40) / a.rows) return RLS_ERR_SHAPE;
    const Span to = matrix(out, a.rows, a.n, ld_out, element), from = matrix(a.logits, a.rows, a.n, a.ld, element);
    if (to.meets(from) && !(out == a.logits && (ld_out == a.ld || a.rows == 1))) return RLS_ERR_SHAPE;
    return check_apart({to}, read);
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int64_t rls_token_logprobs_workspace_bytes(int64_t rows, int64_t n_choices, int32_t top)
{
    if (rows < 1 || rows > RLS_MAX_N || n_choices < 1 || n_choices > RLS_MAX_CHOICES || top < 0 || top > RLS_MAX_TOP) return RLS_ERR_INVALID_ARG;
    return cut_of(rows, n_choices, top).total;
}

int32_t rls_token_logprobs(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits, const int32_t *token_dev,
                           const float *temperature_dev, int32_t top, float *logprob_dev, float *entropy_dev, float *top_logprob_dev,
                           int32_t *top_token_dev, float *norm_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int32_t rc = check_rows(logits_dev, logits_type, rows, n_choices, ld_logits);
    if (rc != RLS_OK) return rc;
    if (top < 0 || top > RLS_MAX_TOP) return RLS_ERR_INVALID_ARG;
    if (!token_dev != !logprob_dev || (top > 0 && (!top_logprob_dev || !top_token_dev))) return RLS_ERR_NULL;
    const int64_t need = rls_token_logprobs_workspace_bytes(rows, n_choices, top);
    rc = check_space(need, workspace_dev, workspace_bytes);
    if (rc != RLS_OK) return rc;
    const int64_t listed = rows * top * 4;
    rc = check_apart({{logprob_dev, rows * 4}, {entropy_dev, rows * 4}, {top_logprob_dev, listed}, {top_token_dev, listed}, {norm_dev, rows * 8}, {workspace_dev, need}},
                     {matrix(logits_dev, rows, n_choices, ld_logits, type_bytes(logits_type)), {token_dev, rows * 4}, {temperature_dev, rows * 4}});
    if (rc != RLS_OK) return rc;
    RowArgs a{};
    a.logits = logits_dev; a.rows = rows; a.n = n_choices; a.ld = ld_logits;
    a.temperature = temperature_dev; a.token = token_dev; a.logprob = logprob_dev; a.entropy = entropy_dev; a.norm = norm_dev;
    a.top = top; a.top_logprob = top_logprob_dev; a.top_token = top_token_dev;
    RLS_HIP_TRY(forward(logits_type, a, static_cast<char *>(workspace_dev), (hipStream_t)stream));
    return RLS_OK;
}

int32_t rls_token_logprobs_backward(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                                    const int32_t *token_dev, const float *temperature_dev, const float *norm_dev, const float *entropy_dev,
                                    const float *dlogprob_dev, const float *dentropy_dev, void *dlogits_dev, int64_t ld_dlogits, void *stream)
{
    int32_t rc = check_rows(logits_dev, logits_type, rows, n_choices, ld_logits);
    if (rc != RLS_OK) return rc;
    if (!norm_dev || (dlogprob_dev && !token_dev) || (dentropy_dev && !entropy_dev)) return RLS_ERR_NULL;
    GradArgs g{};
    g.row.logits = logits_dev; g.row.rows = rows; g.row.n = n_choices; g.row.ld = ld_logits;
    g.row.temperature = temperature_dev; g.row.token = token_dev;
    g.row.norm = const_cast<float *>(norm_dev); g.row.entropy = const_cast<float *>(entropy_dev);
    g.by_logprob = dlogprob_dev; g.by_entropy = dentropy_dev; g.out = dlogits_dev; g.ld_out = ld_dlogits;
    rc = check_gradients(g.row, type_bytes(logits_type), dlogits_dev, ld_dlogits,
                         {{token_dev, rows * 4}, {temperature_dev, rows * 4}, {norm_dev, rows * 8}, {entropy_dev, rows * 4}, {dlogprob_dev, rows * 4}, {dentropy_dev, rows * 4}});
    if (rc != RLS_OK) return rc;
    RLS_HIP_TRY(backward(logits_type, g, (hipStream_t)stream));
    return RLS_OK;
}

int64_t rls_distill_loss_workspace_bytes(int64_t rows, int64_t n_choices)
{
    return rls_token_logprobs_workspace_bytes(rows, n_choices, 0);
}

int32_t rls_distill_loss(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits, const int32_t *teacher_token_dev,
                         const void *teacher_logits_dev, int32_t teacher_type, int32_t k, const float *temperature_dev, float *loss_dev, float *norm_dev,
                         void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int32_t rc = check_rows(logits_dev, logits_type, rows, n_choices, ld_logits);
    if (rc != RLS_OK) return rc;
    if (!teacher_token_dev || !teacher_logits_dev || !loss_dev) return RLS_ERR_NULL;
    if (!is_type(teacher_type) || k < 1 || k > RLS_MAX_TOP) return RLS_ERR_INVALID_ARG;
    const int64_t need = rls_distill_loss_workspace_bytes(rows, n_choices);
    rc = check_space(need, workspace_dev, workspace_bytes);
    if (rc != RLS_OK) return rc;
    rc = check_apart({{loss_dev, rows * 4}, {norm_dev, rows * 8}, {workspace_dev, need}},
                     {matrix(logits_dev, rows, n_choices, ld_logits, type_bytes(logits_type)), {teacher_token_dev, rows * k * 4},
                      {teacher_logits_dev, rows * k * type_bytes(teacher_type)}, {temperature_dev, rows * 4}});
    if (rc != RLS_OK) return rc;
    RowArgs a{};
    a.logits = logits_dev; a.rows = rows; a.n = n_choices; a.ld = ld_logits;
    a.temperature = temperature_dev; a.token = teacher_token_dev; a.logprob = loss_dev; a.norm = norm_dev;
    a.teacher = teacher_logits_dev; a.k = k; a.teacher_type = teacher_type;
    RLS_HIP_TRY(forward(logits_type, a, static_cast<char *>(workspace_dev), (hipStream_t)stream));
    return RLS_OK;
}

int32_t rls_distill_loss_backward(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                                  const int32_t *teacher_token_dev, const void *teacher_logits_dev, int32_t teacher_type, int32_t k,
                                  const float *temperature_dev, const float *norm_dev, const float *dloss_dev, void *dlogits_dev, int64_t ld_dlogits,
                                  void *stream)
{
    int32_t rc = check_rows(logits_dev, logits_type, rows, n_choices, ld_logits);
    if (rc != RLS_OK) return rc;
    if (!teacher_token_dev || !teacher_logits_dev || !norm_dev || !dloss_dev) return RLS_ERR_NULL;
    if (!is_type(teacher_type) || k < 1 || k > RLS_MAX_TOP) return RLS_ERR_INVALID_ARG;
    GradArgs g{};
    g.row.logits = logits_dev; g.row.rows = rows; g.row.n = n_choices; g.row.ld = ld_logits;
    g.row.temperature = temperature_dev; g.row.token = teacher_token_dev; g.row.norm = const_cast<float *>(norm_dev);
    g.row.teacher = teacher_logits_dev; g.row.k = k; g.row.teacher_type = teacher_type;
    g.by_logprob = dloss_dev; g.out = dlogits_dev; g.ld_out = ld_dlogits;
    rc = check_gradients(g.row, type_bytes(logits_type), dlogits_dev, ld_dlogits,
                         {{teacher_token_dev, rows * k * 4}, {teacher_logits_dev, rows * k * type_bytes(teacher_type)}, {temperature_dev, rows * 4},
                          {norm_dev, rows * 8}, {dloss_dev, rows * 4}});
    if (rc != RLS_OK) return rc;
    RLS_HIP_TRY(backward(logits_type, g, (hipStream_t)stream));
    return RLS_OK;
}

}  // extern "C"
