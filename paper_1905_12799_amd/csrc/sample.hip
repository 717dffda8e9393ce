// A draw per row of logits with temperature, top-k, top-p and min-p (rls.h gives the rules): a workgroup per row.
//
// With d = (x - x_max) / temperature every rule is a cut in the order of descending d, equal ones by index.  -d is not
// negative, so its bits order like it does, and the cut is a key (the bits of -d) and an index: an entry is kept if its key is
// smaller, or equal and its index not greater.  Keys and indices are found by bisection, with a count or a sum of weights over
// the row each; weights are whole numbers, so the sums do not depend on who adds what.
#include "element_types.h"
#include "rls_internal.h"

namespace rls {

namespace {

constexpr int kSampleThreads = 256;
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

// sum over the workgroup, the same in every thread
__device__ inline uint64_t group_sum(uint64_t x, uint64_t *lds)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor((unsigned long long)x, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    uint64_t sum = 0;
    for (int w = 0; w < kSampleThreads / 64; ++w) sum += lds[w];
    return sum;
}

// weight of an entry: exp(d) in multiples of 2^-38 (adding 1.5 * 2^14 leaves the whole number in the low bits of a double)
__device__ inline uint64_t weight_of(float e)
{
    constexpr double kMagic = 1.5 * 16384.0;
    return (uint64_t)(__double_as_longlong((double)e + kMagic) - __double_as_longlong(kMagic));
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleArgs p)
{
    __shared__ uint64_t lds[kSampleThreads / 64];
    const int64_t n = p.n;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *const x = static_cast<const T *>(p.logits) + row * p.ld;
        auto logit = [&](int64_t i) {
            const float v = (float)x[i];
            return v == v ? v : -INFINITY;
        };
        float top = -INFINITY;
        for (int64_t i = threadIdx.x; i < n; i += kSampleThreads) top = fmaxf(top, logit(i));
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __float_as_uint(top);
        __syncthreads();
        for (int w = 0; w < kSampleThreads / 64; ++w) top = fmaxf(top, __uint_as_float((uint32_t)lds[w]));
        if (top == -INFINITY) {
            if (threadIdx.x == 0) {
                p.token[row] = -1;
                if (p.logprob) p.logprob[row] = -INFINITY;
            }
            continue;
        }
        float inv = 1.0f;
        int64_t k = p.top_k && p.top_k[row] >= 1 ? min((int64_t)p.top_k[row], n) : n;
        if (p.temperature) {
            const float t = p.temperature[row];
            if (t > 0.0f) inv = 1.0f / t;
            else k = 1;
        }
        auto scaled = [&](int64_t i) {                  // d
            const float v = logit(i), gap = v - top;
            return v == top ? 0.0f : (gap == -INFINITY ? -INFINITY : gap * inv);
        };
        auto key_of = [&](float d) { return __float_as_uint(d) & 0x7fffffffu; };
        // sum over the row of `what(key, weight, index)`
        auto over_row = [&](auto what) {
            uint64_t s = 0;
            for (int64_t i = threadIdx.x; i < n; i += kSampleThreads) {
                const float d = scaled(i);
                s += what(key_of(d), d, i);
            }
            return group_sum(s, lds);
        };
        uint32_t cut = 0x7fffffffu;                     // entries with smaller keys are kept,
        uint64_t ties = ~0ull;                          // and so many with this one
        if (k < n) {
            uint32_t lo = 0, hi = kMaskedKey;           // the smallest key up to which there are k entries
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (over_row([&](uint32_t key, float, int64_t) { return (uint64_t)(key <= mid); }) >= (uint64_t)k) hi = mid;
                else lo = mid + 1;
            }
            cut = lo;
            ties = (uint64_t)k - over_row([&](uint32_t key, float, int64_t) { return (uint64_t)(key < cut); });
        }
        const float p_row = p.top_p ? p.top_p[row] : 1.0f;
        if (p_row < 1.0f) {
            const uint64_t before = over_row([&](uint32_t key, float d, int64_t) { return key < cut ? weight_of(expf(d)) : 0; });
            const uint64_t at_cut = over_row([&](uint32_t key, float, int64_t) { return (uint64_t)(key == cut); });
            const uint64_t w_cut = weight_of(expf(-__uint_as_float(cut)));
            const uint64_t total = before + (cut < kMaskedKey ? w_cut * min(ties, at_cut) : 0);
            const double limit = (double)p_row * (double)total;
            uint32_t lo = 0, hi = cut;                  // the largest key before which there is less than the limit
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                if ((double)over_row([&](uint32_t key, float d, int64_t) { return key < mid ? weight_of(expf(d)) : 0; }) < limit) lo = mid;
                else hi = mid - 1;
            }
            const uint64_t below = over_row([&](uint32_t key, float d, int64_t) { return key < lo ? weight_of(expf(d)) : 0; });
            const uint64_t w = lo < kMaskedKey ? weight_of(expf(-__uint_as_float(lo))) : 0;
            // of the entries with this key as many as begin below the limit, one at least
            uint64_t m = ~0ull;
            if (w > 0) {
                const double estimate = (limit - (double)below) / (double)w;
                m = estimate > 1.0 ? (uint64_t)estimate : 1;
                while (m > 1 && (double)(below + (m - 1) * w) >= limit) --m;
                while ((double)(below + m * w) < limit && m < (uint64_t)n) ++m;
            }
            if (lo < cut) { cut = lo; ties = m; }
            else ties = min(ties, m);
        }
        int64_t last = n - 1;                           // of the entries with the cut's key the ones up to this index
        if (cut <= kMaskedKey && ties < (uint64_t)n) {
            int64_t lo = 0, hi = n - 1;
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (over_row([&](uint32_t key, float, int64_t i) { return (uint64_t)(key == cut && i <= mid); }) >= ties) hi = mid;
                else lo = mid + 1;
            }
            last = lo;
        }
        const float least = p.min_p ? p.min_p[row] : 0.0f;
        auto kept = [&](uint32_t key, float d, int64_t i) -> uint64_t {
            if (key >= kMaskedKey || key > cut || (key == cut && i > last)) return 0;
            const float e = expf(d);
            return e < least && key != 0 ? 0 : weight_of(e);
        };
        const uint64_t total = over_row(kept);
        const float u = p.uniform[row];
        const double mark = (u > 0.0f ? (double)u : 0.0) * (double)total;
        // the first index up to which there is more than the mark, or all
        int64_t lo = 0, hi = n - 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            const uint64_t s = over_row([&](uint32_t key, float d, int64_t i) { return i <= mid ? kept(key, d, i) : 0; });
            if ((double)s > mark || s == total) hi = mid;
            else lo = mid + 1;
        }
        if (threadIdx.x == 0) {
            p.token[row] = (int32_t)lo;
            if (p.logprob) p.logprob[row] = scaled(lo) - logf((float)((double)total * 0x1p-38));
        }
    }
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int64_t rls_sample_workspace_bytes(int64_t rows, int64_t n_choices)
{
    if (rows < 1 || rows > RLS_MAX_N || n_choices < 1 || n_choices > RLS_MAX_CHOICES) return RLS_ERR_INVALID_ARG;
    return 0;
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
    const dim3 grid((unsigned)(rows < 65536 ? rows : 65536)), threads(kSampleThreads);
    const hipStream_t s = (hipStream_t)stream;
    if (logits_type == RLS_F32) hipLaunchKernelGGL(sample_kernel<float>, grid, threads, 0, s, p);
    else if (logits_type == RLS_BF16) hipLaunchKernelGGL(sample_kernel<__bf16>, grid, threads, 0, s, p);
    else hipLaunchKernelGGL(sample_kernel<_Float16>, grid, threads, 0, s, p);
    RLS_HIP_TRY(hipGetLastError());
    return RLS_OK;
}

}  // extern "C"
