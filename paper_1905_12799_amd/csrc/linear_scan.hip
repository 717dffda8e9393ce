// The gated linear recurrence h_t = a_t h_{t-1} + b_t and its backward pass (rls.h gives the formulas).
//
// Steps compose: two in a row are h -> A h + H with A = a' a and H = a' b + b', and a step that was reset is h -> H, whatever h
// (a flag, not A = 0, so that infinities and NaN stay before it).  The backward pass is the same recurrence against time:
// r_t = a_t (dh_t + r_{t+1}) is what step t hands back, the gradients are g_t = dh_t + r_{t+1}, da_t = g_t h_{t-1}.
//
// Memory bounds it: two or three operations for every 2 to 4 bytes.  So every array is read once, in rows of a cache line and
// more, with many loads under way:
// - A workgroup takes a tile, a strip of channels through a stretch of time, and keeps it in registers: a thread V channels of
//   8 or 16 steps in a row, lanes side by side in a line of channels, the others further on in time.  Threads compose their steps, a
//   scan over the lanes and one over the waves (through LDS) compose the tile; what comes before it is looked up from the tiles
//   before (below), and every thread goes through its steps again from the state it then knows.
// - With one channel that lies step by step, the lanes lie along time, 16 bytes of steps each.
// - A few steps over many channels (the step of a single token): a thread per channel.
//
// Tiles of a sequence publish their compositions, and the state after them once they know it (a composition that is a reset); a tile
// looks at those before it, a window of 8 to 256 at a time, back to the nearest state, and takes that state through the compositions
// after it, one by one.  That is how each of them gets its own state, so the result does not depend on where a tile finds one (a single-pass
// scan with look-back, Merrill and Garland 2016; they let compositions join as they come).  An item is one 64-bit word that is written
// and read atomically and is all ones until then, so that no fence is needed (which would write the second-level cache back,
// 100 us here).  A tile that has waited too long for another goes through all the tiles before it by itself, in the same way, so that no
// order in which workgroups run can hold up a call.  (Composed by a launch of their own, chunks of time had their inputs read twice:
// 64 x 262144 returns 138 us, 1 x 65521 x 1024 in bf16 246 us; now 63 and 138, the floors 42 and 104.  The backward pass of
// 8 x 4093 x 2048 in bf16 takes 154 us, 4.4 TB/s.  A launch that clears the items first is 5 us of it, with the gap after it 10.)
//
// Products of gates above 1, and what is added up under them, can pass the largest number where the states themselves do not (gates of 4
// over a state of 0), or be no number.  A composition of that kind is not used: the tile's steps are taken one by one from the
// state before it, thread after thread, and the tile publishes that a state will follow and nothing else.  (64 x 262144 with an infinity
// every 300 steps and resets: 2.5 ms.)
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "element_types.h"
#include "rls_internal.h"
#include "wave.h"

namespace rls {

namespace {

constexpr int kScanThreads = 64;
constexpr int64_t kMostStates = (int64_t)1 << 30;

struct ScanArgs {
    int64_t batch, steps, channels;
    int32_t reverse;
    const float *h0;
    const uint8_t *reset;
    const float *in;                // forward: unused; backward: dh_last or null
    float *out;                     // forward: h_last; backward: dh0 (or null)
    rls_sequence a, h;
    rls_sequence b;                 // forward: the inputs; backward: dh
    rls_sequence da, db;            // backward only
};

template <typename T, typename G>
__global__ void __launch_bounds__(kScanThreads) scan_kernel(ScanArgs p)
{
    const int64_t e = (int64_t)blockIdx.x * kScanThreads + threadIdx.x;
    if (e >= p.batch * p.channels) return;
    const int64_t n = e / p.channels, c = e % p.channels;
    const G *const a = static_cast<const G *>(p.a.data_dev) + n * p.a.batch_stride + c;
    const T *const b = static_cast<const T *>(p.b.data_dev) + n * p.b.batch_stride + c;
    T *const h = static_cast<T *>(p.h.data_dev) + n * p.h.batch_stride + c;
    const uint8_t *const reset = p.reset ? p.reset + n * p.steps : nullptr;
    float s = p.h0 ? p.h0[e] : 0.0f;
    for (int64_t i = 0; i < p.steps; ++i) {
        const int64_t t = p.reverse ? p.steps - 1 - i : i;
        const float x = (float)b[t * p.b.step_stride];
        s = reset && reset[t] ? x : (float)a[t * p.a.step_stride] * s + x;
        h[t * p.h.step_stride] = (T)s;
    }
    if (p.out) p.out[e] = s;
}

template <typename T, typename G>
__global__ void __launch_bounds__(kScanThreads) scan_backward_kernel(ScanArgs p)
{
    const int64_t e = (int64_t)blockIdx.x * kScanThreads + threadIdx.x;
    if (e >= p.batch * p.channels) return;
    const int64_t n = e / p.channels, c = e % p.channels;
    const G *const a = static_cast<const G *>(p.a.data_dev) + n * p.a.batch_stride + c;
    const T *const dh = static_cast<const T *>(p.b.data_dev) + n * p.b.batch_stride + c;
    const T *const h = static_cast<const T *>(p.h.data_dev) + n * p.h.batch_stride + c;
    G *const da = static_cast<G *>(p.da.data_dev) + n * p.da.batch_stride + c;
    T *const db = static_cast<T *>(p.db.data_dev) + n * p.db.batch_stride + c;
    const uint8_t *const reset = p.reset ? p.reset + n * p.steps : nullptr;
    const float h0 = p.h0 ? p.h0[e] : 0.0f;
    float back = p.in ? p.in[e] : 0.0f;             // what the steps after this one hand back
    for (int64_t i = p.steps - 1; i >= 0; --i) {
        const int64_t t = p.reverse ? p.steps - 1 - i : i, before = p.reverse ? t + 1 : t - 1;
        const float g = (float)dh[t * p.b.step_stride] + back;
        const bool cut = reset && reset[t];
        db[t * p.db.step_stride] = (T)g;
        da[t * p.da.step_stride] = (G)(cut ? 0.0f : g * (i == 0 ? h0 : (float)h[before * p.h.step_stride]));
        back = cut ? 0.0f : (float)a[t * p.a.step_stride] * g;
    }
    if (p.out) p.out[e] = back;
}

// ---- tiles --------------------------------------------------------------------------------------

// Of a workgroup; of a strip at most.  (8 waves: 1 x 65521 x 1024 forward 140 -> 144 us, 8 x 4093 x 2048 backward 156 -> 166; strips of
// 16 lanes: 138, 168.  A tile's fixed costs - a barrier, a look at the tiles before, 2 to 4 us each - hide behind another workgroup's loads.)
constexpr int kWaves = 4, kStripLanes = 32;
constexpr int kSteps = 16, kWideSteps = 8;          // of a thread: of two bytes each, of four (16 of those spill registers and are as fast)
constexpr int kAlongWaves = 8, kAlongParts = 2;     // one channel: parts of 64 x 4 steps that a wave takes (4 and 4: 64 x 262144 70 us, 8 and 4: 69, 8 and 2: 61)
constexpr int64_t kAlongTile = (int64_t)kAlongWaves * kAlongParts * 256;
constexpr long long kPatience = 200000;             // ticks of the 100 MHz clock: 2 ms
constexpr int kWindows = 4;                         // that a look keeps; further back it begins anew, where states have come nearer by then

// How the work of a call is cut.
struct ScanCut {
    int32_t lanes;                  // side by side along the channels (a power of two); the other 64 / lanes of a wave are further on in time
    int32_t strips, n_tiles;        // along the channels, along time
    uint64_t *items;                // [batch][n_tiles][strips][channels of a thread][lanes]: what a wave reads at a time lies side by side (32 bytes a lane, four times as much came)
    float *start;                   // [batch][channels] the states before the first step (a copy: the last ones may be written over them)
    long long patience;
};

// An item: A in the high half, H in the low one.  A state, or a composition that no state goes through, has kCut for A; kLater says that there is
// no composition, but that a state will follow.
constexpr uint64_t kEmpty = ~0ull;
constexpr uint32_t kNone = 0xffffffffu, kLater = 0xfffffffeu, kCut = 0xfffffffdu;
__device__ inline uint32_t gate_of(uint64_t item) { return (uint32_t)(item >> 32); }
__device__ inline bool is_state(uint64_t item) { return gate_of(item) == kCut; }
__device__ inline uint64_t state_item(float H) { return (uint64_t)kCut << 32 | __float_as_uint(H); }
__device__ inline bool finite(float x) { return fabsf(x) < INFINITY; }
__device__ inline uint64_t item_of(float A, float H, bool cut)
{
    const uint32_t a = fabsf(H) + (cut ? 0.0f : fabsf(A)) < INFINITY ? (cut ? kCut : __float_as_uint(A)) : kLater;
    return (uint64_t)a << 32 | __float_as_uint(H);
}
// whether a state that compositions give has been lost on the way: it is not finite, and no state before them is to blame
__device__ inline bool lost(float x, float past, bool cut) { return !finite(x) && (cut || finite(past)); }
__device__ inline void publish(uint64_t *at, uint64_t item) { __hip_atomic_store(at, item, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline uint64_t look(const uint64_t *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// a state after the steps of an item
__device__ inline float through(uint64_t item, float x)
{
    const float H = __uint_as_float((uint32_t)item);
    return is_state(item) ? H : fmaf(__uint_as_float(gate_of(item)), x, H);
}

__global__ void __launch_bounds__(256) scan_clear_kernel(ScanCut q, int64_t items, const float *from, int64_t states)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)gridDim.x * 256;
    for (int64_t k = i; k < items; k += n) q.items[k] = kEmpty;
    for (int64_t k = i; k < states; k += n) q.start[k] = from ? from[k] : 0.0f;
}

template <typename T, int N>
struct Pack {
    T x[N];
};
// N elements at any place that an element may lie at
template <typename T, int N>
__device__ inline Pack<T, N> read_pack(const T *p)
{
    Pack<T, N> v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
template <typename T, int N>
__device__ inline void write_pack(T *p, const Pack<T, N> &v)
{
    __builtin_memcpy(p, &v, sizeof(v));
}

// The same as they came: elements of 16 bits stay two to a register until they are used
template <typename T, int V>
struct Raw {
    static constexpr int kWords = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[kWords];
    __device__ inline void read(const T *p)
    {
        w[kWords - 1] = 0;
        __builtin_memcpy(w, p, V * sizeof(T));
    }
    // elements that are all x
    __device__ inline void fill(bool where, float x)
    {
        T both[4 / sizeof(T)];
        for (auto &e : both) e = (T)x;
        uint32_t word;
        __builtin_memcpy(&word, both, 4);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = where ? word : w[i];
    }
    __device__ inline float of(int v) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[v]);
        else if constexpr (std::is_same_v<T, __bf16>) return __uint_as_float(v & 1 ? w[v / 2] & 0xffff0000u : w[v / 2] << 16);
        else {
            const uint16_t half = (uint16_t)(v & 1 ? w[v / 2] >> 16 : w[v / 2]);
            return (float)__builtin_bit_cast(T, half);
        }
    }
    // (whatever has been made of the elements is made again)
    __device__ inline void forget()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
};

// A composition of steps per channel; bit v of `cut`: no state goes through channel v's (nowhere, without resets).
template <int V, bool RESET>
struct Steps {
    float A[V], H[V];
    uint32_t cut;
    static constexpr uint32_t kAll = (1u << V) - 1;
    __device__ inline void clear()
    {
#pragma unroll
        for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
        cut = 0;
    }
    __device__ inline bool is_cut(int v) const { return RESET && (cut >> v & 1u); }
    __device__ inline float of(int v, float x) const { return is_cut(v) ? H[v] : fmaf(A[v], x, H[v]); }
    // not finite (or next to the largest number) where an A or H is not
    __device__ inline float size() const
    {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) sum += fabsf(A[v]) + fabsf(H[v]);
        return sum;
    }
    // these steps after others
    __device__ inline void after(const Steps &o)
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            H[v] = of(v, o.H[v]);
            A[v] *= o.A[v];
        }
        if (RESET) cut |= o.cut;
    }
};

// V channels x kSteps or kWideSteps steps per thread.  Positions i count in the direction of the recurrence, position i is step t = i or steps - 1 - i.
template <typename T, typename G, int V, bool BACK, bool RESET>
__global__ void __launch_bounds__(64 * kWaves, 2) scan_strip_kernel(ScanArgs p, ScanCut q)
{
    constexpr int L = sizeof(T) == 4 ? kWideSteps : kSteps;
    __shared__ float2 totals[2][kWaves][kStripLanes * V];       // compositions of the waves, per channel of the strip
    __shared__ uint32_t total_cut[2][kWaves][kStripLanes];
    __shared__ uint64_t seen[kWindows][kWaves * 64 * V];        // items of the tiles before: [n_groups][V][lanes]
    __shared__ uint32_t states_at[2][kWaves][V];                // a bit per lane of the strip
    __shared__ int gave_up[2][kWaves], large[2][kWaves];
    __shared__ float chain[kStripLanes * V];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lanes = q.lanes, groups = 64 / lanes;             // of a wave, along time
    const int at = lane & (lanes - 1), group = wave * groups + lane / lanes, n_groups = kWaves * groups;
    const int tile = n_groups * L;
    int64_t id = blockIdx.x;
    const int strip = (int)(id % q.strips);
    id /= q.strips;
    const int64_t n = id % p.batch, k = id / p.batch;           // (earlier tiles are in earlier workgroups)
    const int64_t C = p.channels, steps = p.steps;
    // the last strip's lanes take the last V channels where theirs would end beyond; they write their own ones only
    const int64_t c_own = ((int64_t)strip * lanes + at) * V, c0 = max(min(c_own, C - V), (int64_t)0);
    const bool idle = c_own >= C, shared = c0 != c_own;
    const bool down = BACK ? !p.reverse : p.reverse != 0;       // positions run against the steps
    const int64_t i_begin = k * tile, i = i_begin + (int64_t)group * L;
    const bool whole = i_begin + tile < steps;                  // (the one after the last position is read too)
    const G *const a = static_cast<const G *>(p.a.data_dev) + n * p.a.batch_stride + c0;
    const T *const b = static_cast<const T *>(p.b.data_dev) + n * p.b.batch_stride + c0;
    T *const h = static_cast<T *>(p.h.data_dev) + n * p.h.batch_stride + c0;
    const uint8_t *const reset = RESET ? p.reset + n * steps : nullptr;
    auto step_of = [&](int64_t j) { return down ? steps - 1 - j : j; };

    Raw<G, V> a_in[L];
    Raw<T, V> b_in[L], h_in[BACK ? L : 1];                     // (backward: h one step earlier in time)
    uint32_t cut_in;                                            // a bit per step
    // a row of each step from position `from` on
    auto rows_of = [&](const auto *base, int64_t stride, int64_t from, auto &rows) {
        using E = std::remove_cv_t<std::remove_pointer_t<decltype(base)>>;
        if (whole) {
            const E *first = base + step_of(from) * stride;
            const int64_t next = down ? -stride : stride;
#pragma unroll
            for (int j = 0; j < L; ++j) {
                rows[j].read(first);
                first += next;
            }
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) rows[j].read(base + step_of(min(from + j, steps - 1)) * stride);
        }
    };
    rows_of(a, p.a.step_stride, i, a_in);
    rows_of(b, p.b.step_stride, i, b_in);
    cut_in = 0;
    if constexpr (RESET) {
#pragma unroll
        for (int j = 0; j < L; ++j) cut_in |= (reset[step_of(min(i + j, steps - 1))] != 0 ? 1u : 0u) << j;
    }
    if (!whole) {                                               // steps after the last one change nothing
#pragma unroll
        for (int j = 0; j < L; ++j) {
            a_in[j].fill(i + j >= steps, 1.0f);
            b_in[j].fill(i + j >= steps, 0.0f);
        }
        const int64_t left = steps - i;
        cut_in &= left >= L ? ~0u : (left > 0 ? (1u << left) - 1 : 0u);
    }
    // one step more
    auto append = [&](Steps<V, RESET> &s, const Raw<G, V> &gate, const Raw<T, V> &input, bool cut) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float x = gate.of(v), y = input.of(v);
            s.H[v] = BACK ? (cut ? 0.0f : x * (y + s.H[v])) : (cut ? y : fmaf(x, s.H[v], y));
            s.A[v] *= x;
        }
        if (RESET) s.cut = cut ? Steps<V, RESET>::kAll : s.cut;
    };
    // over the groups of a wave that come before a lane's, and its own
    auto scan_wave = [&](Steps<V, RESET> &s) {
        for (int d = lanes; d < 64; d <<= 1) {
            Steps<V, RESET> o;
#pragma unroll
            for (int v = 0; v < V; ++v) { o.A[v] = __shfl_up(s.A[v], d, 64); o.H[v] = __shfl_up(s.H[v], d, 64); }
            o.cut = RESET ? __shfl_up(s.cut, d, 64) : 0u;
            if (lane >= d) s.after(o);
        }
    };
    int turn = 0;                                               // (no wave reads the other half any more: one barrier a time)
    // The compositions of the waves before this one and of all; whether any composition on the way cannot be used (the same in every thread: every wave
    // has all channels of the strip).  Without resets what is not finite stays so, and is seen at the end.
    auto scan_waves = [&](const Steps<V, RESET> &s, Steps<V, RESET> &before, Steps<V, RESET> &all) {
        if constexpr (RESET) {
            const bool any = __any(!(s.size() < INFINITY));
            if (lane == 0) large[turn][wave] = any;
        }
        if (lane >= 64 - lanes) {
#pragma unroll
            for (int v = 0; v < V; ++v) totals[turn][wave][at * V + v] = make_float2(s.A[v], s.H[v]);
            if (RESET) total_cut[turn][wave][at] = s.cut;
        }
        __syncthreads();
        before.clear();
        all.clear();
        float size = 0.0f;
        int odd = 0;
#pragma unroll 2                                                // (all at once, they are 64 registers)
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) before = all;
            Steps<V, RESET> o;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 x = totals[turn][w][at * V + v];
                o.A[v] = x.x;
                o.H[v] = x.y;
            }
            o.cut = RESET ? total_cut[turn][w][at] : 0u;
            o.after(all);
            all = o;
            if constexpr (RESET) {
                size += all.size();
                odd |= large[turn][w];
            }
        }
        if (!RESET) size = all.size();
        turn ^= 1;
        return odd != 0 || __any(!(size < INFINITY)) != 0;
    };

    const int64_t row = (int64_t)q.strips * V * lanes;          // items of a tile of time
    uint64_t *const items = q.items + n * q.n_tiles * row + (int64_t)strip * V * lanes + at;
    const float *const start = q.start + n * C + c0;
    const bool tells = group == 0 && k + 1 < q.n_tiles;
    // The states before the tile, from what the tiles before it publish; false if one of them is missing for too long (the same in every thread)
    auto look_back = [&](float (&x)[V]) {
        const uint32_t all_lanes = lanes == 32 ? ~0u : (1u << lanes) - 1;
        uint32_t known[V];                                      // a bit per lane: a state is among what was seen
        int64_t end = k;
        int windows = 0;
        for (int flip = 0;; flip ^= 1) {
            if (windows == 0) {
#pragma unroll
                for (int v = 0; v < V; ++v) known[v] = 0;
            }
            const int64_t other = end - n_groups + group;
            uint64_t item[V];
            bool missing = false;
#pragma unroll
            for (int v = 0; v < V; ++v) item[v] = item_of(1.0f, 0.0f, false);
            if (other >= 0) {
                const long long since = wall_clock64();
                for (;;) {
                    uint32_t most = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        item[v] = look(items + other * row + v * lanes);
                        most = max(most, gate_of(item[v]));
                    }
                    missing = most == kNone;
                    // (a tile that says "later" is running: for it there is no limit)
                    if (most < kLater || (missing && wall_clock64() - since >= q.patience)) break;
                    __builtin_amdgcn_s_sleep(4);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                seen[windows][(group * V + v) * lanes + at] = item[v];
                uint64_t states = __ballot(is_state(item[v]));
                for (int d = 32; d >= lanes; d >>= 1) states |= states >> d;
                if (lane == 0) states_at[flip][wave][v] = (uint32_t)states & all_lanes;
            }
            const bool any = __any(missing);
            if (lane == 0) gave_up[flip][wave] = any;
            __syncthreads();
            bool all_known = true;
            int failed = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int w = 0; w < kWaves; ++w) known[v] |= (uint32_t)__builtin_amdgcn_readfirstlane((int)states_at[flip][w][v]);
                all_known &= known[v] == all_lanes;
            }
#pragma unroll
            for (int w = 0; w < kWaves; ++w) failed |= gave_up[flip][w];
            if (failed) return false;
            ++windows;
            if (all_known) break;                               // (tile 0 publishes nothing but its state)
            end -= n_groups;
            if (windows == kWindows) {
                windows = 0;
                end = k;
                __builtin_amdgcn_s_sleep(16);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = 0.0f;                // (a state takes its place)
        for (int w = windows - 1; w >= 0; --w) {
            const uint64_t *const of_window = &seen[w][at];
#pragma unroll 4
            for (int g = 0; g < n_groups; ++g) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = through(of_window[(g * V + v) * lanes], x[v]);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) sum += fabsf(x[v]);
        bool good = sum < INFINITY;
        while (__builtin_expect(!good, 0)) {                    // the state that the tile before has (it is running, as all are that published something)
            good = true;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint64_t item = look(items + (k - 1) * row + v * lanes);
                x[v] = __uint_as_float((uint32_t)item);
                good &= is_state(item);
            }
            if (!good) __builtin_amdgcn_s_sleep(4);
        }
        return true;
    };
    // The states before each thread and after the tile, step by step, from position `first` of the thread on.  (All of the workgroup together.  Rare, so
    // the rows are read again: kept for this as well they are registers of every call.)
    auto one_by_one = [&](const float (&from)[V], int64_t first, float (&x)[V], float (&end)[V]) {
        for (int g = 0; g < n_groups; ++g) {
            __syncthreads();
            if (group != g) continue;
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = end[v] = g == 0 ? from[v] : chain[at * V + v];
#pragma unroll 1
            for (int j = 0; j < L; ++j) {
                if (first + j >= steps) break;
                const int64_t t = step_of(first + j);
                Raw<G, V> gate;
                Raw<T, V> input;
                gate.read(a + t * p.a.step_stride);
                input.read(b + t * p.b.step_stride);
                const bool cut = RESET && reset[t] != 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float e = gate.of(v), y = input.of(v);
                    end[v] = BACK ? (cut ? 0.0f : e * (y + end[v])) : (cut ? y : fmaf(e, end[v], y));
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) chain[at * V + v] = end[v];
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) end[v] = chain[at * V + v];
    };

    Steps<V, RESET> own, waves_before, of_tile;
    float past[V];                                              // the states before the tile
#pragma unroll
    for (int v = 0; v < V; ++v) past[v] = 0.0f;
    if (k == 0) {                                               // (before any barrier: the last state may be written over it, by another wave)
        const float *const from = q.n_tiles > 1 ? q.start : (BACK ? p.in : p.h0);
#pragma unroll
        for (int v = 0; v < V; ++v) past[v] = from && c0 + v < C ? from[n * C + c0 + v] : 0.0f;
    }
    own.clear();
#pragma unroll
    for (int j = 0; j < L; ++j) append(own, a_in[j], b_in[j], RESET && (cut_in >> j & 1u));
    scan_wave(own);
    const bool odd = scan_waves(own, waves_before, of_tile);
    if (k > 0) {
        if (tells) {
#pragma unroll
            for (int v = 0; v < V; ++v) publish(items + k * row + v * lanes, item_of(of_tile.A[v], of_tile.H[v], of_tile.is_cut(v)));
        }
        if (__builtin_expect(!look_back(past), 0)) {            // through all the tiles before, all of the workgroup together
#pragma unroll
            for (int v = 0; v < V; ++v) past[v] = c0 + v < C ? start[v] : 0.0f;
            for (int64_t j0 = (int64_t)group * L; j0 < i_begin; j0 += tile) {
                Steps<V, RESET> s, unused, other;
                s.clear();
#pragma unroll 2
                for (int j = 0; j < L; ++j) {
                    const int64_t t = step_of(j0 + j);
                    Raw<G, V> gate;
                    Raw<T, V> input;
                    gate.read(a + t * p.a.step_stride);
                    input.read(b + t * p.b.step_stride);
                    append(s, gate, input, RESET && reset[t] != 0);
                }
                scan_wave(s);
                float x[V], end[V];
                const bool strange = scan_waves(s, unused, other);
                if (strange) one_by_one(past, j0, x, end);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float then = other.of(v, past[v]);
                    past[v] = strange && lost(then, past[v], other.is_cut(v)) ? end[v] : then;
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float then = of_tile.of(v, past[v]);
        if (tells && !(odd && lost(then, past[v], of_tile.is_cut(v)))) publish(items + k * row + v * lanes, state_item(then));
    }
    float x[V];                                                 // the state before the thread's steps
    Steps<V, RESET> before;
#pragma unroll
    for (int v = 0; v < V; ++v) { before.A[v] = __shfl_up(own.A[v], lanes, 64); before.H[v] = __shfl_up(own.H[v], lanes, 64); }
    before.cut = RESET ? __shfl_up(own.cut, lanes, 64) : 0u;
    if (lane < lanes) before.clear();
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = before.of(v, waves_before.of(v, past[v]));
    if (__builtin_expect(odd, 0)) {
        float y[V], end[V];
        one_by_one(past, i, y, end);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (tells && lost(of_tile.of(v, past[v]), past[v], of_tile.is_cut(v))) publish(items + k * row + v * lanes, state_item(end[v]));
            x[v] = lost(x[v], past[v], before.is_cut(v) || waves_before.is_cut(v)) ? y[v] : x[v];
        }
    }
    if constexpr (BACK) rows_of(static_cast<const T *>(h), p.h.step_stride, i + 1, h_in);
    G *const da = BACK ? static_cast<G *>(p.da.data_dev) + n * p.da.batch_stride + c0 : nullptr;
    T *const to = (BACK ? static_cast<T *>(p.db.data_dev) + n * p.db.batch_stride : static_cast<T *>(p.h.data_dev) + n * p.h.batch_stride) + c0;
    const int64_t first = step_of(i), next = down ? -1 : 1;
    T *out_row = to + first * (BACK ? p.db.step_stride : p.h.step_stride);
    const int64_t out_next = next * (BACK ? p.db.step_stride : p.h.step_stride);
    G *out_row_a = BACK ? da + first * p.da.step_stride : nullptr;
    const int64_t out_next_a = BACK ? next * p.da.step_stride : 0;
#pragma unroll
    for (int j = 0; j < L; ++j) { a_in[j].forget(); b_in[j].forget(); }
#pragma unroll
    for (int j = 0; j < L; ++j) {
        if (!whole && i + j >= steps) break;
        Pack<T, V> out;
        Pack<G, V> out_a;
        const bool cut = RESET && (cut_in >> j & 1u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float g = a_in[j].of(v), e = b_in[j].of(v);
            if constexpr (BACK) {
                const float y = e + x[v];
                float prev = h_in[j].of(v);
                if (!whole && i + j == steps - 1) prev = p.h0 && c0 + v < C ? p.h0[n * C + c0 + v] : 0.0f;
                out_a.x[v] = (G)(cut ? 0.0f : y * prev);
                out.x[v] = (T)y;
                x[v] = cut ? 0.0f : g * y;
            } else {
                x[v] = cut ? e : fmaf(g, x[v], e);
                out.x[v] = (T)x[v];
            }
        }
        if (!idle) {
            if (!shared) {
                write_pack<T, V>(out_row, out);
                if constexpr (BACK) write_pack<G, V>(out_row_a, out_a);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (c0 + v >= c_own) {
                        out_row[v] = out.x[v];
                        if constexpr (BACK) out_row_a[v] = out_a.x[v];
                    }
            }
        }
        out_row += out_next;
        if constexpr (BACK) out_row_a += out_next_a;
        if (!whole && i + j == steps - 1 && p.out && !idle) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (c0 + v >= c_own) p.out[n * C + c0 + v] = x[v];
        }
    }
}

// One channel, its steps side by side: a wave takes kAlongParts parts of 64 x 4 steps, a lane four of each.
template <typename T, typename G, bool BACK, bool RESET>
__global__ void __launch_bounds__(64 * kAlongWaves) scan_along_kernel(ScanArgs p, ScanCut q)
{
    constexpr int P = kAlongParts, L = 4;
    __shared__ float2 totals[kAlongWaves];
    __shared__ int total_cut[kAlongWaves];
    __shared__ uint64_t seen[kWindows][64];         // items of the tiles before (the first wave's)
    __shared__ float found, chain;
    __shared__ bool gave_up;
    __shared__ int large[kAlongWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n = blockIdx.x % p.batch, k = blockIdx.x / p.batch, steps = p.steps;
    const bool down = BACK ? !p.reverse : p.reverse != 0;
    const G *const a = static_cast<const G *>(p.a.data_dev) + n * p.a.batch_stride;
    const T *const b = static_cast<const T *>(p.b.data_dev) + n * p.b.batch_stride;
    const T *const h = static_cast<const T *>(p.h.data_dev) + n * p.h.batch_stride;
    const uint8_t *const reset = RESET ? p.reset + n * steps : nullptr;
    auto step_of = [&](int64_t j) { return down ? steps - 1 - j : j; };
    // four positions, in their order
    auto four = [&](const auto *base, int64_t from, auto &x) {
        using E = std::remove_cv_t<std::remove_pointer_t<decltype(base)>>;
        if (from + L <= steps) {
            const Pack<E, L> v = read_pack<E, L>(base + (down ? steps - L - from : from));
#pragma unroll
            for (int j = 0; j < L; ++j) x[j] = (float)(down ? v.x[L - 1 - j] : v.x[j]);
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) x[j] = (float)base[step_of(min(from + j, steps - 1))];
        }
    };
    float a_in[P][L], b_in[P][L], h_in[BACK ? P : 1][L];
    uint32_t cut_in[P];
    auto compose = [&](int u, Steps<1, RESET> &s) {
        s.clear();
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const bool cut = RESET && (cut_in[u] >> j & 1u);
            const float x = a_in[u][j], y = b_in[u][j];
            s.H[0] = BACK ? (cut ? 0.0f : x * (y + s.H[0])) : (cut ? y : fmaf(x, s.H[0], y));
            s.A[0] *= x;
            if (RESET) s.cut = cut ? 1u : s.cut;
        }
    };
    // over the lanes before, and the lane's own
    auto scan_lanes = [&](Steps<1, RESET> &s) {
        auto move = [&](auto ctrl, auto rows) {
            constexpr int c = decltype(ctrl)::value, m = decltype(rows)::value;
            Steps<1, RESET> o;
            o.A[0] = lane_move<c, m>(1.0f, s.A[0]);
            o.H[0] = lane_move<c, m>(0.0f, s.H[0]);
            o.cut = RESET ? lane_move<c, m>(0u, s.cut) : 0u;
            s.after(o);
        };
        using std::integral_constant;
        move(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());
        move(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
        move(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
        move(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
        move(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());
        move(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());
    };
    auto of_last_lane = [&](const Steps<1, RESET> &s) {
        Steps<1, RESET> o;
        o.A[0] = last_lane(s.A[0]);
        o.H[0] = last_lane(s.H[0]);
        o.cut = last_lane(s.cut);
        return o;
    };
    uint64_t *const items = q.items + n * q.n_tiles;
    // The state before the tile, from what the tiles before it publish (by one wave); false if one of them is missing for too long
    auto look_back = [&](float &x) {
        int64_t end = k;
        int windows = 0, first;
        for (;;) {
            const int64_t other = end - 64 + lane;
            uint64_t item = item_of(1.0f, 0.0f, false);
            bool missing = false;
            if (other >= 0) {
                const long long since = wall_clock64();
                for (;;) {
                    item = look(items + other);
                    missing = gate_of(item) == kNone;
                    // (a tile that says "later" is running: for it there is no limit)
                    if (gate_of(item) < kLater || (missing && wall_clock64() - since >= q.patience)) break;
                    __builtin_amdgcn_s_sleep(4);
                }
            }
            if (__any(missing)) return false;
            seen[windows++][lane] = item;
            const uint64_t states = __ballot(is_state(item));
            if (states != 0) {                      // (tile 0 publishes nothing but its state)
                first = 63 - __clzll((long long)states);
                break;
            }
            end -= 64;
            if (windows == kWindows) {
                windows = 0;
                end = k;
                __builtin_amdgcn_s_sleep(16);
            }
        }
        __builtin_amdgcn_wave_barrier();            // (a wave's accesses to LDS stay in their order)
        x = 0.0f;                                   // (a state takes its place)
        for (int w = windows - 1; w >= 0; --w, first = 0) {
#pragma unroll 4
            for (int l = first; l < 64; ++l) x = through(seen[w][l], x);
        }
        while (__builtin_expect(!finite(x), 0)) {   // the state that the tile before has (it is running, as all are that published something)
            const uint64_t item = look(items + k - 1);
            x = __uint_as_float((uint32_t)item);
            if (is_state(item)) break;
            x = INFINITY;
            __builtin_amdgcn_s_sleep(4);
        }
        return true;
    };
    // The states before a lane's steps of each part, and after the tile, step by step: lane after lane.  (All of the workgroup together.)
    auto one_by_one = [&](float from, float (&x)[P]) {
        for (int w = 0; w < kAlongWaves; ++w) {
            __syncthreads();
            if (wave != w) continue;
            float y = w == 0 ? from : chain;
#pragma unroll
            for (int u = 0; u < P; ++u)
                for (int l = 0; l < 64; ++l) {
                    x[u] = lane == l ? y : x[u];
                    float z = y;
#pragma unroll
                    for (int j = 0; j < L; ++j) {
                        const bool cut = RESET && (cut_in[u] >> j & 1u);
                        z = BACK ? (cut ? 0.0f : a_in[u][j] * (b_in[u][j] + z)) : (cut ? b_in[u][j] : fmaf(a_in[u][j], z, b_in[u][j]));
                    }
                    y = __shfl(z, l, 64);
                }
            if (lane == 0) chain = y;
        }
        __syncthreads();
        return chain;
    };
    Steps<1, RESET> own[P], before, all;            // per part: the wave's steps up to the lane's; the waves before; the tile
    float past = 0.0f;                              // the state before the tile
    if (k == 0) {                                   // (before any barrier: the last state may be written over it, by another wave)
        const float *const from = q.n_tiles > 1 ? q.start : (BACK ? p.in : p.h0);
        past = from ? from[n] : 0.0f;
    }
    int64_t i0;                                     // the lane's first position; part u begins 64 * L further on
    bool known = k == 0, odd;
    // once, or through all the tiles before the own one first
    for (int64_t here = k;;) {
        const int64_t i_begin = here * kAlongTile;
        const bool whole = i_begin + kAlongTile < steps;
        i0 = i_begin + (wave * P * 64 + lane) * L;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int64_t from = i0 + u * 64 * L;
            four(a, from, a_in[u]);
            four(b, from, b_in[u]);
            cut_in[u] = 0;
            if constexpr (RESET) {
                float r[L];
                four(reset, from, r);
#pragma unroll
                for (int j = 0; j < L; ++j) cut_in[u] |= (r[j] != 0.0f ? 1u : 0u) << j;
            }
            if (!whole) {                           // steps after the last one change nothing
#pragma unroll
                for (int j = 0; j < L; ++j) {
                    a_in[u][j] = from + j < steps ? a_in[u][j] : 1.0f;
                    b_in[u][j] = from + j < steps ? b_in[u][j] : 0.0f;
                }
                const int64_t left = steps - from;
                cut_in[u] &= left >= L ? ~0u : (left > 0 ? (1u << left) - 1 : 0u);
            }
        }
        Steps<1, RESET> of_wave;
        of_wave.clear();
#pragma unroll
        for (int u = 0; u < P; ++u) {
            compose(u, own[u]);
            scan_lanes(own[u]);
            Steps<1, RESET> part = of_last_lane(own[u]);
            own[u].after(of_wave);
            part.after(of_wave);
            of_wave = part;
        }
        if constexpr (RESET) {                      // (without resets what is not finite stays so, and is seen at the end)
            float size = 0.0f;
#pragma unroll
            for (int u = 0; u < P; ++u) size += own[u].size();
            const bool any = __any(!(size < INFINITY));
            if (lane == 0) large[wave] = any;
        }
        if (lane == 0) {
            totals[wave] = make_float2(of_wave.A[0], of_wave.H[0]);
            total_cut[wave] = of_wave.cut;
        }
        __syncthreads();
        before.clear();
        all.clear();
        float size = 0.0f;
        int not_small = 0;
#pragma unroll
        for (int w = 0; w < kAlongWaves; ++w) {
            if (w == wave) before = all;
            Steps<1, RESET> o;
            o.A[0] = totals[w].x;
            o.H[0] = totals[w].y;
            o.cut = total_cut[w];
            o.after(all);
            all = o;
            if constexpr (RESET) {
                size += all.size();
                not_small |= large[w];
            }
        }
        if (!RESET) size = all.size();
        odd = not_small != 0 || !(size < INFINITY);         // a composition on the way cannot be used (the same in every thread)
        if (here == k && known) break;
        if (here == k && wave == 0) {
            if (lane == 0) publish(items + k, item_of(all.A[0], all.H[0], all.is_cut(0)));
            float x = 0.0f;
            const bool there = look_back(x);
            if (lane == 0) {
                found = x;
                gave_up = !there;
            }
        }
        __syncthreads();                            // (nor are the totals read any more)
        if (here < k) {
            const float then = all.of(0, past);
            float x[P], end = 0.0f;
            if (odd) end = one_by_one(past, x);
            past = odd && lost(then, past, all.is_cut(0)) ? end : then;
            known = ++here == k;
        } else {
            past = found;
            if (!gave_up) break;                    // (the same in every thread)
            here = 0;
            past = q.start[n];
        }
    }
    if constexpr (BACK) {
#pragma unroll
        for (int u = 0; u < P; ++u) four(h, i0 + u * 64 * L + 1, h_in[u]);
    }
    const float after = all.of(0, past);
    const bool late = odd && lost(after, past, all.is_cut(0));
    if (threadIdx.x == 0 && k + 1 < q.n_tiles && !late) publish(items + k, state_item(after));
    const float of_waves = before.of(0, past);
    G *const da = BACK ? static_cast<G *>(p.da.data_dev) + n * p.da.batch_stride : nullptr;
    T *const to = BACK ? static_cast<T *>(p.db.data_dev) + n * p.db.batch_stride : static_cast<T *>(p.h.data_dev) + n * p.h.batch_stride;
    float first[P];                                 // the state before the lane's steps of a part
    uint32_t cuts = RESET && before.cut ? (1u << P) - 1 : 0u;        // a bit per part: no state goes through what comes before it in the tile
    {
        Steps<1, RESET> parts_before;               // of the wave
        parts_before.clear();
#pragma unroll
        for (int u = 0; u < P; ++u) {
            Steps<1, RESET> o;
            o.A[0] = __shfl_up(own[u].A[0], 1, 64);
            o.H[0] = __shfl_up(own[u].H[0], 1, 64);
            o.cut = RESET ? __shfl_up(own[u].cut, 1, 64) : 0u;
            if (lane == 0) o = parts_before;
            first[u] = o.of(0, of_waves);
            if (RESET) cuts |= o.cut << u;
            parts_before = of_last_lane(own[u]);
        }
    }
    if (__builtin_expect(odd, 0)) {
        float y[P];
        const float end = one_by_one(past, y);
        if (threadIdx.x == 0 && k + 1 < q.n_tiles && late) publish(items + k, state_item(end));
#pragma unroll
        for (int u = 0; u < P; ++u) first[u] = lost(first[u], past, cuts >> u & 1u) ? y[u] : first[u];
    }
#pragma unroll
    for (int u = 0; u < P; ++u) {
        const int64_t i = i0 + u * 64 * L;
        float x = first[u];
        float y[L], ya[L];
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const bool cut = RESET && (cut_in[u] >> j & 1u);
            if constexpr (BACK) {
                y[j] = b_in[u][j] + x;
                const float prev = i + j < steps - 1 ? h_in[u][j] : (p.h0 ? p.h0[n] : 0.0f);
                ya[j] = cut ? 0.0f : y[j] * prev;
                x = cut ? 0.0f : a_in[u][j] * y[j];
            } else {
                x = cut ? b_in[u][j] : fmaf(a_in[u][j], x, b_in[u][j]);
                y[j] = x;
            }
            if (i + j == steps - 1 && p.out) p.out[n] = x;
        }
        auto put = [&](auto *where, const float (&z)[L]) {
            using E = std::remove_pointer_t<decltype(where)>;
            if (i + L <= steps) {
                Pack<E, L> v;
#pragma unroll
                for (int j = 0; j < L; ++j) v.x[j] = (E)(down ? z[L - 1 - j] : z[j]);
                write_pack<E, L>(where + (down ? steps - L - i : i), v);
            } else {
#pragma unroll
                for (int j = 0; j < L; ++j)
                    if (i + j < steps) where[step_of(i + j)] = (E)z[j];
            }
        };
        put(to, y);
        if constexpr (BACK) put(da, ya);
    }
}

// ---- which way a call takes ----------------------------------------------------------------------

// Up to so many steps a thread goes through a channel by itself; a thread | tiles, in bf16, forward: 64 x 16 x 4096 12 | 25 us, 4 x 64 x 4096 19 | 13.
// Many channels hide a thread's waits for longer: 1024 x 32 x 1024 53 | 90 us, 1024 x 64 x 1024 168 | 122, and one channel's tile is
// 4096 steps: 100000 x 64 x 1 181 | 543, 100000 x 200 x 1 744 | 550.
int64_t few_steps(int64_t states, bool along) { return along && states >= (1 << 16) ? 128 : (states >= (1 << 17) ? 32 : 16); }

thread_local long long g_patience = kPatience;

struct ScanPlan {
    bool tiles, along;
    int vec;                                        // channels of a thread
    ScanCut cut;
    int64_t items, bytes;
};

ScanPlan plan_scan(int64_t batch, int64_t steps, int64_t channels, bool wide, bool unit_steps)
{
    ScanPlan r{};
    r.along = channels == 1 && unit_steps;
    r.vec = channels >= 4 ? 4 : 1;
    int lanes = 1;
    while (lanes < kStripLanes && lanes * r.vec < channels) lanes *= 2;
    r.cut.lanes = lanes;
    r.cut.strips = (int32_t)((channels + lanes * r.vec - 1) / (lanes * r.vec));
    const int64_t tile = r.along ? kAlongTile : (int64_t)kWaves * (64 / lanes) * (wide ? kWideSteps : kSteps);
    const int64_t tiles = std::max<int64_t>(1, (steps + tile - 1) / tile);
    r.tiles = steps > few_steps(batch * channels, r.along) && batch * r.cut.strips <= ((int64_t)1 << 22) / tiles;
    if (!r.tiles) return r;
    r.cut.n_tiles = (int32_t)tiles;
    if (tiles > 1) {
        r.items = batch * tiles * r.cut.strips * lanes * r.vec;
        r.bytes = align_up(r.items * 8, 256) + align_up(batch * channels * 4, 256);
    }
    return r;
}

template <typename T, typename G, bool BACK, bool RESET>
void launch_tiles(const ScanArgs &p, const ScanPlan &plan, hipStream_t s)
{
    const dim3 grid((unsigned)(p.batch * plan.cut.strips * plan.cut.n_tiles));
    if (plan.along) hipLaunchKernelGGL((scan_along_kernel<T, G, BACK, RESET>), grid, dim3(64 * kAlongWaves), 0, s, p, plan.cut);
    else if (plan.vec == 1) hipLaunchKernelGGL((scan_strip_kernel<T, G, 1, BACK, RESET>), grid, dim3(64 * kWaves), 0, s, p, plan.cut);
    else hipLaunchKernelGGL((scan_strip_kernel<T, G, 4, BACK, RESET>), grid, dim3(64 * kWaves), 0, s, p, plan.cut);
}

template <typename T, typename G>
hipError_t launch_scan(const ScanArgs &p, const ScanPlan &plan, bool backward, hipStream_t s)
{
    if (plan.tiles) {
        if (plan.items > 0) {
            const int64_t states = p.batch * p.channels, most = std::max(plan.items, states);
            hipLaunchKernelGGL(scan_clear_kernel, dim3((unsigned)std::min<int64_t>((most + 1023) / 1024, 2048)), dim3(256), 0, s, plan.cut, plan.items,
                               backward ? p.in : p.h0, states);
        }
        if (backward) p.reset ? launch_tiles<T, G, true, true>(p, plan, s) : launch_tiles<T, G, true, false>(p, plan, s);
        else p.reset ? launch_tiles<T, G, false, true>(p, plan, s) : launch_tiles<T, G, false, false>(p, plan, s);
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)((p.batch * p.channels + kScanThreads - 1) / kScanThreads);
    if (backward) hipLaunchKernelGGL((scan_backward_kernel<T, G>), dim3(blocks), dim3(kScanThreads), 0, s, p);
    else hipLaunchKernelGGL((scan_kernel<T, G>), dim3(blocks), dim3(kScanThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_scan_of_type(const rls_scan_shape &shape, const ScanArgs &p, const ScanPlan &plan, bool backward, hipStream_t s)
{
    if (shape.type == RLS_F32) return launch_scan<float, float>(p, plan, backward, s);
    if (shape.type == RLS_BF16)
        return shape.gate_type == RLS_F32 ? launch_scan<__bf16, float>(p, plan, backward, s) : launch_scan<__bf16, __bf16>(p, plan, backward, s);
    return shape.gate_type == RLS_F32 ? launch_scan<_Float16, float>(p, plan, backward, s) : launch_scan<_Float16, _Float16>(p, plan, backward, s);
}

bool sizes_fit(int64_t batch, int64_t steps, int64_t channels)
{
    return batch >= 1 && batch <= kMostStates && channels >= 1 && channels <= kMostStates && batch <= kMostStates / channels && steps >= 0 &&
           steps <= RLS_MAX_N;
}

int32_t check_shape(const rls_scan_shape *shape)
{
    if (!shape) return RLS_ERR_NULL;
    if (!sizes_fit(shape->batch, shape->steps, shape->channels)) return RLS_ERR_INVALID_ARG;
    if (!is_type(shape->type) || (shape->gate_type != RLS_F32 && shape->gate_type != shape->type)) return RLS_ERR_INVALID_ARG;
    return RLS_OK;
}

// Strides of an array that is read may be anything that is not negative; one that is written must not overlap itself.
int32_t check_sequence(const rls_scan_shape &shape, const rls_sequence *q, bool written)
{
    if (!q) return RLS_ERR_NULL;
    if (shape.steps > 0 && !q->data_dev) return RLS_ERR_NULL;
    if (q->batch_stride < 0 || q->step_stride < 0) return RLS_ERR_SHAPE;
    if (!written) return RLS_OK;
    // channels lie innermost, then either the steps of a sequence side by side or the sequences of a step
    const int64_t c = shape.channels, t = shape.steps, n = shape.batch;
    const bool steps_inner = (t <= 1 || q->step_stride >= c) && (n == 1 || q->batch_stride >= (t <= 1 ? c : (t - 1) * q->step_stride + c));
    const bool batch_inner = (n == 1 || q->batch_stride >= c) && (t <= 1 || q->step_stride >= (n == 1 ? c : (n - 1) * q->batch_stride + c));
    return steps_inner || batch_inner ? RLS_OK : RLS_ERR_SHAPE;
}

// Where an array lies: rows of so many bytes, repeated at one or two distances.
struct Place {
    int64_t at, width;
    struct { int64_t count, apart; } inner, outer;
    int64_t end() const { return at + (inner.count - 1) * inner.apart + (outer.count - 1) * outer.apart + width; }
};
Place place_of(const void *data, int64_t bytes) { return Place{(int64_t)(uintptr_t)data, data ? bytes : 0, {1, 0}, {1, 0}}; }
Place place_of(const rls_scan_shape &shape, const rls_sequence &q, int64_t element)
{
    Place r = place_of(q.data_dev, shape.steps > 0 ? shape.channels * element : 0);
    r.inner = {shape.steps, q.step_stride * element};
    r.outer = {shape.batch, q.batch_stride * element};
    if (r.inner.apart > r.outer.apart) std::swap(r.inner, r.outer);
    for (auto *d : {&r.inner, &r.outer}) {
        if (r.width == 0 || d->apart == 0) d->count = 1;
        // rows that touch are one
        if (d->apart <= r.width && (d == &r.inner || r.inner.count == 1)) {
            r.width += (d->count - 1) * d->apart;
            d->count = 1;
        }
        if (d->count == 1) d->apart = 0;
    }
    return r;
}

// Whether two arrays have a byte in common.  Views of one buffer may lie between each other's rows: with the same distances that is found out
// exactly; where they have more than two distances between them, arrays that reach into each other count as common.
bool overlap(const Place &x, const Place &y)
{
    if (x.width == 0 || y.width == 0 || x.end() <= y.at || y.end() <= x.at) return false;
    int64_t apart[4], n = 0;
    for (const auto &d : {x.inner, x.outer, y.inner, y.outer})
        if (d.count > 1) apart[n++] = d.apart;
    std::sort(apart, apart + n);
    n = std::unique(apart, apart + n) - apart;
    if (n > 2) return true;
    // y's rows less x's are i * near + j * far apart, with each of these between the two ends
    auto ends = [&](int64_t of, int64_t *least, int64_t *most) {
        *least = *most = 0;
        for (const auto &d : {x.inner, x.outer})
            if (d.count > 1 && d.apart == of) *least -= d.count - 1;
        for (const auto &d : {y.inner, y.outer})
            if (d.count > 1 && d.apart == of) *most += d.count - 1;
    };
    auto down = [](int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); };
    const int64_t near = n > 0 ? apart[0] : 1, far = n > 1 ? apart[1] : 1;
    int64_t i0 = 0, i1 = 0, j0 = 0, j1 = 0;
    if (n > 0) ends(near, &i0, &i1);
    if (n > 1) ends(far, &j0, &j1);
    // a byte is common where they are less than x's width ahead, less than y's behind
    const int64_t d = y.at - x.at, lo = -y.width + 1 - d, hi = x.width - 1 - d;
    j0 = std::max(j0, down(lo - i1 * near + far - 1, far));
    j1 = std::min(j1, down(hi - i0 * near, far));
    if (j1 - j0 > 1000) return true;                // (windows of one array that overlap each other, many deep)
    for (int64_t j = j0; j <= j1; ++j)
        if (std::max(i0, down(lo - j * far + near - 1, near)) <= std::min(i1, down(hi - j * far, near))) return true;
    return false;
}

// nothing that is written may lie in anything else; a state may take another one's place as a whole
int32_t check_overlap(std::initializer_list<Place> written, std::initializer_list<Place> read)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (const Place &r : read)
            if (overlap(*w, r)) return RLS_ERR_SHAPE;
        for (auto v = written.begin(); v != w; ++v)
            if (overlap(*w, *v)) return RLS_ERR_SHAPE;
    }
    return RLS_OK;
}

int32_t plan_call(const rls_scan_shape &shape, bool unit_steps, void *workspace, int64_t bytes, ScanPlan *plan)
{
    if (rls_linear_scan_workspace_bytes(shape.batch, shape.steps, shape.channels) > 0) {
        if (!workspace || (uintptr_t)workspace % 256 != 0) return RLS_ERR_WORKSPACE;
        if (bytes < rls_linear_scan_workspace_bytes(shape.batch, shape.steps, shape.channels)) return RLS_ERR_WORKSPACE;
    }
    *plan = plan_scan(shape.batch, shape.steps, shape.channels, shape.type == RLS_F32, unit_steps);
    plan->cut.patience = g_patience;
    if (plan->items > 0) {
        plan->cut.items = static_cast<uint64_t *>(workspace);
        plan->cut.start = reinterpret_cast<float *>(static_cast<char *>(workspace) + align_up(plan->items * 8, 256));
    }
    return RLS_OK;
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int32_t rls_scan_wait_limit(int64_t ticks)
{
    g_patience = ticks < 0 ? kPatience : ticks;
    return RLS_OK;
}

int32_t rls_scan_overlap(const rls_scan_shape *shape, const rls_sequence *x, int32_t x_type, const rls_sequence *y, int32_t y_type)
{
    return overlap(place_of(*shape, *x, type_bytes(x_type)), place_of(*shape, *y, type_bytes(y_type))) ? 1 : 0;
}

int64_t rls_linear_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t channels)
{
    if (!sizes_fit(batch, steps, channels)) return RLS_ERR_INVALID_ARG;
    int64_t most = 0;                               // (of any type and any strides)
    for (int form = 0; form < 4; ++form) most = std::max(most, plan_scan(batch, steps, channels, (form & 1) != 0, (form & 2) != 0).bytes);
    return most;
}

int32_t rls_linear_scan(const rls_scan_shape *shape, const rls_sequence *a, const rls_sequence *b, const float *h0_dev,
                        const uint8_t *reset_dev, const rls_sequence *h, float *h_last_dev, void *workspace_dev,
                        int64_t workspace_bytes, void *stream)
{
    int32_t rc = check_shape(shape);
    if (rc == RLS_OK) rc = check_sequence(*shape, a, false);
    if (rc == RLS_OK) rc = check_sequence(*shape, b, false);
    if (rc == RLS_OK) rc = check_sequence(*shape, h, true);
    if (rc != RLS_OK) return rc;
    const bool unit = a->step_stride == 1 && b->step_stride == 1 && h->step_stride == 1;
    ScanPlan plan;
    rc = plan_call(*shape, unit, workspace_dev, workspace_bytes, &plan);
    if (rc != RLS_OK) return rc;
    const int64_t wide = type_bytes(shape->type), gate = type_bytes(shape->gate_type), states = shape->batch * shape->channels * 4;
    const Place none{}, start = place_of(h0_dev, states), last = place_of(h_last_dev, states), flags = place_of(reset_dev, shape->batch * shape->steps);
    rc = check_overlap({place_of(*shape, *h, wide), last}, {place_of(*shape, *a, gate), place_of(*shape, *b, wide), flags});
    if (rc == RLS_OK) rc = check_overlap({place_of(*shape, *h, wide), h_last_dev == h0_dev ? none : last}, {start});
    if (rc != RLS_OK) return rc;
    ScanArgs p{};
    p.batch = shape->batch; p.steps = shape->steps; p.channels = shape->channels; p.reverse = shape->reverse;
    p.h0 = h0_dev; p.reset = reset_dev; p.out = h_last_dev;
    p.a = *a; p.b = *b; p.h = *h;
    RLS_HIP_TRY(launch_scan_of_type(*shape, p, plan, false, (hipStream_t)stream));
    return RLS_OK;
}

int32_t rls_linear_scan_backward(const rls_scan_shape *shape, const rls_sequence *a, const rls_sequence *h, const rls_sequence *dh,
                                 const float *h0_dev, const uint8_t *reset_dev, const float *dh_last_dev, const rls_sequence *da,
                                 const rls_sequence *db, float *dh0_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int32_t rc = check_shape(shape);
    if (rc == RLS_OK) rc = check_sequence(*shape, a, false);
    if (rc == RLS_OK) rc = check_sequence(*shape, h, false);
    if (rc == RLS_OK) rc = check_sequence(*shape, dh, false);
    if (rc == RLS_OK) rc = check_sequence(*shape, da, true);
    if (rc == RLS_OK) rc = check_sequence(*shape, db, true);
    if (rc != RLS_OK) return rc;
    const bool unit = a->step_stride == 1 && h->step_stride == 1 && dh->step_stride == 1 && da->step_stride == 1 && db->step_stride == 1;
    ScanPlan plan;
    rc = plan_call(*shape, unit, workspace_dev, workspace_bytes, &plan);
    if (rc != RLS_OK) return rc;
    const int64_t wide = type_bytes(shape->type), gate = type_bytes(shape->gate_type), states = shape->batch * shape->channels * 4;
    const Place none{}, start = place_of(h0_dev, states), last = place_of(dh_last_dev, states), first = place_of(dh0_dev, states),
                flags = place_of(reset_dev, shape->batch * shape->steps), to_a = place_of(*shape, *da, gate), to_b = place_of(*shape, *db, wide);
    rc = check_overlap({to_a, to_b, first}, {place_of(*shape, *a, gate), place_of(*shape, *h, wide), place_of(*shape, *dh, wide), start, flags});
    if (rc == RLS_OK) rc = check_overlap({to_a, to_b, dh0_dev == dh_last_dev ? none : first}, {last});
    if (rc != RLS_OK) return rc;
    ScanArgs p{};
    p.batch = shape->batch; p.steps = shape->steps; p.channels = shape->channels; p.reverse = shape->reverse;
    p.h0 = h0_dev; p.reset = reset_dev; p.in = dh_last_dev; p.out = dh0_dev;
    p.a = *a; p.b = *dh; p.h = *h; p.da = *da; p.db = *db;
    RLS_HIP_TRY(launch_scan_of_type(*shape, p, plan, true, (hipStream_t)stream));
    return RLS_OK;
}

}  // extern "C"
