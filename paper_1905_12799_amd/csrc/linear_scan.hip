// The gated linear recurrence h_t = a_t h_{t-1} + b_t and its backward pass (rls.h gives the formulas).
//
// Steps compose: two in a row are h -> A h + H with A = a' a and H = a' b + b', and a step that was reset is h -> H, whatever h
// (a flag, not A = 0, so that infinities and NaN stay before it).  The backward pass is the same recurrence against time:
// r_t = a_t (dh_t + r_{t+1}) is what step t hands back, the gradients are g_t = dh_t + r_{t+1}, da_t = g_t h_{t-1}.
//
// Memory bounds it: two or three operations for every 2 to 4 bytes.  So every array is to be read once, in rows of a cache
// line and more, with many loads under way:
// - A workgroup takes a strip of channels of one sequence through time in tiles; a thread takes V channels (16 bytes) of L
//   steps in a row, lanes side by side in a line of channels, the others further on in time.  A tile stays in registers:
//   threads compose their steps, a scan over the lanes and one over the waves (through LDS, one barrier) give each the state
//   it starts from, and it goes through its steps again.  The next tile's loads are issued before that.
// - With one channel the lanes lie along time, and a thread's steps are what it loads 16 bytes at a time.
// - Where strips are too few to fill the chip, time is cut into chunks: a launch composes each chunk's steps, a second one goes
//   through the chunks from the states that the earlier ones' compositions give.  The inputs are read twice then.
// - A few steps over many channels (the step of a single token): a thread per channel.
#include <algorithm>

#include "element_types.h"
#include "rls_internal.h"

namespace rls {

namespace {

constexpr int kScanThreads = 64;
constexpr int kWaves = 8;                           // of a workgroup that goes through tiles
constexpr int kMostChunks = 256;
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

// How the work of a call is cut.  Chunk k's composition is item k + 1 of its sequence, item 0 the state before the first step.
struct ScanCut {
    int32_t lanes;                  // side by side along the channels (a power of two); the other 64 / lanes of a wave are further on in time
    int32_t strips, n_chunks;
    int64_t chunk;                  // steps
    float2 *items;                  // [batch][n_chunks][channels] (A, H); of the last chunk no item is needed
    int32_t *cuts;                  // [batch][strips][n_chunks] whether A is a reset
};

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

// WHOLE: the tiles of a sequence one after the other.  COMPOSE: a chunk's composition.  APPLY: the tiles of a chunk.
enum { WHOLE, COMPOSE, APPLY };

// V channels x L steps per thread; ALONG: V = 1 and the L steps lie side by side in memory.  Positions i count in the direction of
// the recurrence, position i is step t = i or steps - 1 - i.
template <typename T, typename G, int V, int L, bool ALONG, bool BACK, int MODE>
__global__ void __launch_bounds__(64 * kWaves) scan_tiles_kernel(ScanArgs p, ScanCut q)
{
    extern __shared__ __align__(16) float2 totals[];            // [2][kWaves][lanes * V] compositions of the waves
    __shared__ int wave_cut[2][kWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lanes = q.lanes, groups = 64 / lanes;             // of a wave, along time
    const int at = lane & (lanes - 1), group = wave * groups + lane / lanes;
    const int64_t tile = (int64_t)kWaves * groups * L;
    int64_t id = blockIdx.x;
    const int strip = (int)(id % q.strips);
    id /= q.strips;
    const int64_t n = id % p.batch;
    const int chunk = (int)(id / p.batch);
    const int64_t C = p.channels, steps = p.steps;
    // the last strip's lanes take the last V channels where theirs would end beyond; they write their own ones only
    const int64_t c_own = ((int64_t)strip * lanes + at) * V, c0 = max(min(c_own, C - V), (int64_t)0);
    const bool idle = c_own >= C, shared = c0 != c_own;
    const bool down = BACK ? !p.reverse : p.reverse != 0;       // positions run against the steps
    const int64_t i_begin = (int64_t)chunk * q.chunk, i_end = min(steps, i_begin + q.chunk);
    const G *const a = static_cast<const G *>(p.a.data_dev) + n * p.a.batch_stride + c0;
    const T *const b = static_cast<const T *>(p.b.data_dev) + n * p.b.batch_stride + c0;
    T *const h = static_cast<T *>(p.h.data_dev) + n * p.h.batch_stride + c0;
    G *const da = BACK ? static_cast<G *>(p.da.data_dev) + n * p.da.batch_stride + c0 : nullptr;
    T *const db = BACK ? static_cast<T *>(p.db.data_dev) + n * p.db.batch_stride + c0 : nullptr;
    const uint8_t *const reset = p.reset ? p.reset + n * steps : nullptr;
    auto step_of = [&](int64_t i) { return down ? steps - 1 - i : i; };

    constexpr int N = ALONG ? L : V, M = ALONG ? 1 : L;         // elements of a load, loads of a thread
    Pack<G, N> a_in[M];
    Pack<T, N> b_in[M], h_in[M];                                // (backward: h one step earlier in time)
    uint32_t cut_in;                                            // a bit per step
    // loads of the steps from position i0 on; positions from i_end on repeat the last one
    auto load = [&](int64_t i0) {
        cut_in = 0;
        if constexpr (ALONG) {
            auto fetch = [&](const auto *from, int64_t i, auto &pack) {
                if (i + L <= steps) pack = read_pack<std::remove_cv_t<std::remove_pointer_t<decltype(from)>>, L>(from + (down ? steps - L - i : i));
                else
#pragma unroll
                    for (int j = 0; j < L; ++j) pack.x[down ? L - 1 - j : j] = from[step_of(min(i + j, steps - 1))];
            };
            fetch(a, i0, a_in[0]);
            fetch(b, i0, b_in[0]);
            if constexpr (BACK && MODE != COMPOSE) fetch(static_cast<const T *>(h), i0 + 1, h_in[0]);
            if (reset) {
#pragma unroll
                for (int j = 0; j < L; ++j) cut_in |= (reset[step_of(min(i0 + j, steps - 1))] != 0 ? 1u : 0u) << j;
            }
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int64_t t = step_of(min(i0 + j, steps - 1));
                a_in[j] = read_pack<G, V>(a + t * p.a.step_stride);
                b_in[j] = read_pack<T, V>(b + t * p.b.step_stride);
                if constexpr (BACK && MODE != COMPOSE) h_in[j] = read_pack<T, V>(h + step_of(min(i0 + j + 1, steps - 1)) * p.h.step_stride);
                if (reset) cut_in |= (reset[t] != 0 ? 1u : 0u) << j;
            }
        }
    };
    // element v of step j of a loaded array
    auto element = [&](const auto *packs, int j, int v) {
        if constexpr (ALONG) return (float)(down ? packs[0].x[L - 1 - j] : packs[0].x[j]);
        else return (float)packs[j].x[v];
    };

    // compositions of steps: A, H per channel, and whether they were cut
    struct Steps {
        float A[V], H[V];
        int cut;
    };
    auto nothing = [](Steps &s) {
#pragma unroll
        for (int v = 0; v < V; ++v) { s.A[v] = 1.0f; s.H[v] = 0.0f; }
        s.cut = 0;
    };
    auto apply = [](float A, float H, int cut, float x) { return cut ? H : A * x + H; };
    // s after `first`
    auto compose = [&](Steps &s, const float (&A)[V], const float (&H)[V], int cut) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s.H[v] = apply(s.A[v], s.H[v], s.cut, H[v]);
            s.A[v] = s.A[v] * A[v];
        }
        s.cut |= cut;
    };
    // over the groups of a wave that come before a lane's and, where `own`, its own
    auto scan_wave = [&](Steps &s) {
        for (int d = lanes; d < 64; d <<= 1) {
            Steps o;
#pragma unroll
            for (int v = 0; v < V; ++v) { o.A[v] = __shfl_up(s.A[v], d, 64); o.H[v] = __shfl_up(s.H[v], d, 64); }
            o.cut = __shfl_up(s.cut, d, 64);
            if (lane >= d) compose(s, o.A, o.H, o.cut);
        }
    };
    int turn = 0;
    // the states before this wave's steps and after those of all waves, from `state` before them all
    auto scan_waves = [&](const Steps &s, float (&state)[V], float (&before)[V], Steps *whole) {
        float2 *const t = totals + (size_t)turn * kWaves * lanes * V;
        if (lane >= 64 - lanes) {
#pragma unroll
            for (int v = 0; v < V; ++v) t[(wave * lanes + at) * V + v] = make_float2(s.A[v], s.H[v]);
            if (at == 0) wave_cut[turn][wave] = s.cut;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int cut = wave_cut[turn][w];
            if (w == wave) {
#pragma unroll
                for (int v = 0; v < V; ++v) before[v] = state[v];
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 x = t[(w * lanes + at) * V + v];
                state[v] = apply(x.x, x.y, cut, state[v]);
                if (whole) {
                    whole->H[v] = apply(x.x, x.y, cut, whole->H[v]);
                    whole->A[v] = whole->A[v] * x.x;
                }
            }
            if (whole) whole->cut |= cut;
        }
        turn ^= 1;                                              // (the other half is read by no wave any more: one barrier a time)
    };
    // the steps loaded, from position i0 on, in turn: what(position, j, cut, identity)
    auto step_values = [&](int64_t i, int j, int v, float &x, float &y) {
        const bool in = i + j < i_end;
        const float g = in ? element(a_in, j, v) : 1.0f, e = in ? element(b_in, j, v) : 0.0f;
        const bool cut = cut_in >> j & 1u && in;
        x = cut ? 0.0f : g;
        y = BACK ? (cut ? 0.0f : g * e) : e;
        return cut;
    };
    auto compose_loaded = [&](int64_t i, Steps &s) {
#pragma unroll
        for (int j = 0; j < L; ++j) {
            bool cut = false;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float x, y;
                cut = step_values(i, j, v, x, y);
                s.H[v] = cut ? y : x * s.H[v] + y;
                s.A[v] = s.A[v] * x;
            }
            s.cut |= cut;
        }
    };

    float state[V];                                             // before the next tile, the same in every group
    if (MODE != APPLY) {
        const float *const from = BACK ? p.in : p.h0;
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = from && c0 + v < C ? from[n * C + c0 + v] : 0.0f;
    }
    float2 *const items = MODE == WHOLE ? nullptr : q.items + n * q.n_chunks * C + c0;
    int32_t *const cuts = MODE == WHOLE ? nullptr : q.cuts + (n * q.strips + strip) * q.n_chunks;
    if constexpr (MODE == COMPOSE) {
        // groups take equal parts of the chunk, whole loads of L steps
        const int64_t per = (q.chunk / L + (int64_t)kWaves * groups - 1) / ((int64_t)kWaves * groups) * L;
        const int64_t from = i_begin + per * group, to = min(i_end, from + per);
        Steps s;
        nothing(s);
        for (int64_t i = from; i < to; i += L) {
            load(i);
            compose_loaded(i, s);
        }
        scan_wave(s);
        float before[V], none[V];
        Steps whole;
        nothing(whole);
#pragma unroll
        for (int v = 0; v < V; ++v) none[v] = 0.0f;
        scan_waves(s, none, before, &whole);
        if (group == 0 && !idle) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (c0 + v >= c_own) {
                    if (chunk == 0) items[v] = make_float2(0.0f, state[v]);
                    items[(int64_t)(chunk + 1) * C + v] = make_float2(whole.A[v], whole.H[v]);
                }
            if (at == 0) {
                if (chunk == 0) cuts[0] = 1;
                cuts[chunk + 1] = whole.cut;
            }
        }
        return;
    }
    if constexpr (MODE == APPLY) {
        // the state before the chunk: the items up to it, shared among the groups
        const int per = (chunk + 1 + kWaves * groups - 1) / (kWaves * groups);
        const int from = per * group, to = min(chunk + 1, from + per);
        Steps s;
        nothing(s);
        for (int k = from; k < to; ++k) {
            const int cut = cuts[k];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 x = items[(int64_t)k * C + v];
                s.H[v] = apply(x.x, x.y, cut, s.H[v]);
                s.A[v] = s.A[v] * x.x;
            }
            s.cut |= cut;
        }
        scan_wave(s);
        float before[V];
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = 0.0f;
        scan_waves(s, state, before, nullptr);
    }
    load(i_begin + (int64_t)group * L);
    for (int64_t i0 = i_begin; i0 < i_end; i0 += tile) {
        const int64_t i = i0 + (int64_t)group * L;
        Steps s;
        nothing(s);
        compose_loaded(i, s);
        scan_wave(s);
        float x[V];
        scan_waves(s, state, x, nullptr);
        // the groups before in this wave
        {
            Steps o;
#pragma unroll
            for (int v = 0; v < V; ++v) { o.A[v] = __shfl_up(s.A[v], lanes, 64); o.H[v] = __shfl_up(s.H[v], lanes, 64); }
            o.cut = __shfl_up(s.cut, lanes, 64);
            if (lane >= lanes) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = apply(o.A[v], o.H[v], o.cut, x[v]);
            }
        }
        Pack<T, N> out[M];
        Pack<G, N> out_a[M];
#pragma unroll
        for (int j = 0; j < L; ++j) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float y;
                if constexpr (BACK) {
                    const bool cut = cut_in >> j & 1u;
                    const float g = element(b_in, j, v) + x[v];
                    const float prev = i + j < steps - 1 ? element(h_in, j, v) : (p.h0 && c0 + v < C ? p.h0[n * C + c0 + v] : 0.0f);
                    const float ga = cut ? 0.0f : g * prev;
                    x[v] = cut ? 0.0f : element(a_in, j, v) * g;
                    y = g;
                    if constexpr (ALONG) out_a[0].x[j] = (G)ga;
                    else out_a[j].x[v] = (G)ga;
                } else {
                    x[v] = cut_in >> j & 1u ? element(b_in, j, v) : element(a_in, j, v) * x[v] + element(b_in, j, v);
                    y = x[v];
                }
                if constexpr (ALONG) out[0].x[j] = (T)y;
                else out[j].x[v] = (T)y;
            }
            if (i + j == steps - 1 && p.out && !idle) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (c0 + v >= c_own) p.out[n * C + c0 + v] = x[v];
            }
        }
        const int64_t i_next = i0 + tile + (int64_t)group * L;
        if (i0 + tile < i_end) load(i_next);
        T *const to = BACK ? db : h;
        const int64_t stride = BACK ? p.db.step_stride : p.h.step_stride;
        if constexpr (ALONG) {
            auto put = [&](auto *where, auto &pack) {
                using E = std::remove_pointer_t<decltype(where)>;
                if (down) {
#pragma unroll
                    for (int j = 0; j < L / 2; ++j) { const E y = pack.x[j]; pack.x[j] = pack.x[L - 1 - j]; pack.x[L - 1 - j] = y; }
                }
                if (i + L <= i_end) write_pack<E, L>(where + (down ? steps - L - i : i), pack);
                else
#pragma unroll
                    for (int j = 0; j < L; ++j)
                        if (i + j < i_end) where[step_of(i + j)] = pack.x[down ? L - 1 - j : j];
            };
            if (!idle) {
                put(to, out[0]);
                if constexpr (BACK) put(da, out_a[0]);
            }
        } else if (!idle) {
#pragma unroll
            for (int j = 0; j < L; ++j) {
                if (i + j >= i_end) break;
                const int64_t t = step_of(i + j);
                if (!shared) {
                    write_pack<T, V>(to + t * stride, out[j]);
                    if constexpr (BACK) write_pack<G, V>(da + t * p.da.step_stride, out_a[j]);
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (c0 + v >= c_own) {
                            to[t * stride + v] = out[j].x[v];
                            if constexpr (BACK) da[t * p.da.step_stride + v] = out_a[j].x[v];
                        }
                }
            }
        }
    }
}

// ---- which way a call takes ----------------------------------------------------------------------

constexpr int64_t kFewSteps = 16;
constexpr int64_t kFill = 512;                      // workgroups that fill the chip
constexpr int64_t kAlongSteps = 16, kStripSteps = 4;

struct ScanPlan {
    bool tiles, along;
    int vec;                                        // channels of a thread
    ScanCut cut;
    int64_t bytes;
};

ScanPlan plan_scan(int64_t batch, int64_t steps, int64_t channels, int element_bytes, bool unit_steps)
{
    ScanPlan r{};
    r.along = channels == 1 && unit_steps;
    r.vec = channels >= 16 / element_bytes ? 16 / element_bytes : 1;
    int lanes = 1;
    while (lanes < 128 / element_bytes / r.vec && lanes * r.vec < channels) lanes *= 2;
    r.cut.lanes = lanes;
    r.cut.strips = (int32_t)((channels + lanes * r.vec - 1) / (lanes * r.vec));
    r.cut.n_chunks = 1;
    r.cut.chunk = std::max<int64_t>(steps, 1);
    const int64_t blocks = batch * r.cut.strips;
    r.tiles = steps > kFewSteps && blocks <= ((int64_t)1 << 22);
    if (!r.tiles) return r;
    const int64_t tile = (int64_t)kWaves * (64 / lanes) * (r.along ? kAlongSteps : kStripSteps);
    const int64_t chunks = std::min<int64_t>({kMostChunks, (kFill + blocks - 1) / blocks, (steps + 2 * tile - 1) / (2 * tile)});
    if (blocks < kFill / 2 && chunks > 1) {
        r.cut.chunk = ((steps + chunks - 1) / chunks + tile - 1) / tile * tile;
        r.cut.n_chunks = (int32_t)((steps + r.cut.chunk - 1) / r.cut.chunk);
    }
    if (r.cut.n_chunks > 1)
        r.bytes = align_up(batch * r.cut.n_chunks * channels * 8, 256) + align_up(batch * r.cut.strips * r.cut.n_chunks * 4, 256);
    return r;
}

template <typename T, typename G, int V, int L, bool ALONG>
hipError_t launch_tiles(const ScanArgs &p, const ScanCut &q, bool backward, hipStream_t s)
{
    const dim3 grid((unsigned)(p.batch * q.strips * q.n_chunks)), threads(64 * kWaves);
    const size_t lds = (size_t)2 * kWaves * q.lanes * V * sizeof(float2);
    if (q.n_chunks == 1) {
        if (backward) hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, true, WHOLE>), grid, threads, lds, s, p, q);
        else hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, false, WHOLE>), grid, threads, lds, s, p, q);
        return hipGetLastError();
    }
    const dim3 all_but_last((unsigned)(p.batch * q.strips * (q.n_chunks - 1)));
    if (backward) hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, true, COMPOSE>), all_but_last, threads, lds, s, p, q);
    else hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, false, COMPOSE>), all_but_last, threads, lds, s, p, q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (backward) hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, true, APPLY>), grid, threads, lds, s, p, q);
    else hipLaunchKernelGGL((scan_tiles_kernel<T, G, V, L, ALONG, false, APPLY>), grid, threads, lds, s, p, q);
    return hipGetLastError();
}

template <typename T, typename G>
hipError_t launch_scan(const ScanArgs &p, const ScanPlan &plan, bool backward, hipStream_t s)
{
    if (plan.tiles) {
        if (plan.along) return launch_tiles<T, G, 1, kAlongSteps, true>(p, plan.cut, backward, s);
        if (plan.vec == 1) return launch_tiles<T, G, 1, kStripSteps, false>(p, plan.cut, backward, s);
        return launch_tiles<T, G, 16 / sizeof(T), kStripSteps, false>(p, plan.cut, backward, s);
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

int32_t plan_call(const rls_scan_shape &shape, bool unit_steps, void *workspace, int64_t bytes, ScanPlan *plan)
{
    if (rls_linear_scan_workspace_bytes(shape.batch, shape.steps, shape.channels) > 0) {
        if (!workspace || (uintptr_t)workspace % 256 != 0) return RLS_ERR_WORKSPACE;
        if (bytes < rls_linear_scan_workspace_bytes(shape.batch, shape.steps, shape.channels)) return RLS_ERR_WORKSPACE;
    }
    *plan = plan_scan(shape.batch, shape.steps, shape.channels, type_bytes(shape.type), unit_steps);
    if (plan->bytes > 0) {
        plan->cut.items = static_cast<float2 *>(workspace);
        plan->cut.cuts = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + align_up(shape.batch * plan->cut.n_chunks * shape.channels * 8, 256));
    }
    return RLS_OK;
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int64_t rls_linear_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t channels)
{
    if (!sizes_fit(batch, steps, channels)) return RLS_ERR_INVALID_ARG;
    int64_t most = 0;                               // (of any type and any strides)
    for (int bytes = 2; bytes <= 4; bytes += 2)
        for (int unit = 0; unit < 2; ++unit) most = std::max(most, plan_scan(batch, steps, channels, bytes, unit != 0).bytes);
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
    ScanArgs p{};
    p.batch = shape->batch; p.steps = shape->steps; p.channels = shape->channels; p.reverse = shape->reverse;
    p.h0 = h0_dev; p.reset = reset_dev; p.in = dh_last_dev; p.out = dh0_dev;
    p.a = *a; p.b = *dh; p.h = *h; p.da = *da; p.db = *db;
    RLS_HIP_TRY(launch_scan_of_type(*shape, p, plan, true, (hipStream_t)stream));
    return RLS_OK;
}

}  // extern "C"
