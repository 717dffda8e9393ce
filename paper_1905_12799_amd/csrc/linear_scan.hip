// The gated linear recurrence h_t = a_t h_{t-1} + b_t and its backward pass (rls.h gives the formulas): a thread takes one
// channel of one sequence and goes through the steps.
#include "element_types.h"
#include "rls_internal.h"

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

template <typename T, typename G>
hipError_t launch_scan(const ScanArgs &p, bool backward, hipStream_t s)
{
    const unsigned blocks = (unsigned)((p.batch * p.channels + kScanThreads - 1) / kScanThreads);
    if (backward) hipLaunchKernelGGL((scan_backward_kernel<T, G>), dim3(blocks), dim3(kScanThreads), 0, s, p);
    else hipLaunchKernelGGL((scan_kernel<T, G>), dim3(blocks), dim3(kScanThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_scan_of_type(const rls_scan_shape &shape, const ScanArgs &p, bool backward, hipStream_t s)
{
    if (shape.type == RLS_F32) return launch_scan<float, float>(p, backward, s);
    if (shape.type == RLS_BF16)
        return shape.gate_type == RLS_F32 ? launch_scan<__bf16, float>(p, backward, s) : launch_scan<__bf16, __bf16>(p, backward, s);
    return shape.gate_type == RLS_F32 ? launch_scan<_Float16, float>(p, backward, s) : launch_scan<_Float16, _Float16>(p, backward, s);
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

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int64_t rls_linear_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t channels)
{
    if (!sizes_fit(batch, steps, channels)) return RLS_ERR_INVALID_ARG;
    return 0;
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
    const int64_t need = rls_linear_scan_workspace_bytes(shape->batch, shape->steps, shape->channels);
    if (need > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 256 != 0 || workspace_bytes < need)) return RLS_ERR_WORKSPACE;
    ScanArgs p{};
    p.batch = shape->batch; p.steps = shape->steps; p.channels = shape->channels; p.reverse = shape->reverse;
    p.h0 = h0_dev; p.reset = reset_dev; p.out = h_last_dev;
    p.a = *a; p.b = *b; p.h = *h;
    RLS_HIP_TRY(launch_scan_of_type(*shape, p, false, (hipStream_t)stream));
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
    const int64_t need = rls_linear_scan_workspace_bytes(shape->batch, shape->steps, shape->channels);
    if (need > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 256 != 0 || workspace_bytes < need)) return RLS_ERR_WORKSPACE;
    ScanArgs p{};
    p.batch = shape->batch; p.steps = shape->steps; p.channels = shape->channels; p.reverse = shape->reverse;
    p.h0 = h0_dev; p.reset = reset_dev; p.in = dh_last_dev; p.out = dh0_dev;
    p.a = *a; p.b = *dh; p.h = *h; p.da = *da; p.db = *db;
    RLS_HIP_TRY(launch_scan_of_type(*shape, p, true, (hipStream_t)stream));
    return RLS_OK;
}

}  // extern "C"
