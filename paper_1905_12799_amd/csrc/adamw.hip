// One AdamW step over many tensors: rls_adamw_step (rls.h gives the formulas).
//
// Every array is read once and written once: 28 bytes a parameter with fp32 throughout, 16 in bf16 with master weights and
// 8-bit moments, for some fifteen operations, so memory bounds it: 63 million parameters in fp32 take 344 us (5.1 TB/s, the rate of a
// large copy), 185 million in bf16 with 8-bit moments 633 to 645 us (4.6 TB/s).  One launch takes the tensors of one kind, up to kTensors
// of them: their addresses travel as kernel arguments, and a workgroup finds its own by bisection of the first workgroups'
// numbers.  (A launch per tensor would cost a network of small layers its launches: 2 us each.)
//
// A wave takes 256 consecutive elements at a time, four a lane: that is also the block that shares a scale where the moments
// are held in 8 bits, so that the largest magnitude of a block is one reduction over a wave and nothing goes through LDS.
#include <math.h>

#include "element_types.h"
#include "rls_internal.h"
#include "wave.h"

namespace rls {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamBlock = 256;                   // elements that share a scale
constexpr int kAdamTurns = 4;                     // blocks a wave takes
constexpr int64_t kAdamChunk = (int64_t)kAdamTurns * (kAdamThreads / 64) * kAdamBlock;
constexpr int kTensors = 44;                      // per launch (kernel arguments end at 4 KB)
constexpr uint32_t kAdamGrid = 1u << 23;          // workgroups per launch at most
constexpr int64_t kAdamMost = (int64_t)1 << 34;   // elements of a tensor

struct AdamTensor {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    uint64_t bits;                                // random bits: the state that the tensor's draws start from
    int32_t quads;                                // every array can be reached four elements at a time
};
struct AdamArgs {
    AdamTensor tensor[kTensors];
    uint32_t first[kTensors];                     // first workgroup of each tensor
    int32_t n_tensors;
    double one_less_beta1, one_less_beta2;
    float beta1, beta2, keep, step, root, eps;
    const float *grad_scale;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// the output function of SplitMix64 (Steele, Lea, Flood 2014)
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
__host__ __device__ inline uint64_t mix(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// The scale of a block whose largest magnitude is given: the power of two 2^e that brings it into (224, 448].  A power of two
// costs an 8-bit float nothing (its precision does not depend on where in its range it lies) and makes both ways exact.
__device__ inline int block_exponent(float largest)
{
    const uint32_t u = __float_as_uint(largest);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -120);
}

// |x| / 2^e as an 8-bit float with 4 bits of exponent (bias 7) and 3 of mantissa, rounded up with a probability of 1/65536 times
// what is left below, by `r` of 16 random bits; below 2^-6, where the format's steps stop shrinking, 2^-6 is added first and its
// code taken off again, so that one shift serves all.  What is no finite number becomes the format's NaN.
__device__ inline uint32_t encode(float x, float inv, uint32_t r, uint32_t least)
{
    const float mag = fabsf(x);
    const float y = mag * inv;
    const bool small = y < 0.015625f;
    const uint32_t u = __float_as_uint(small ? y + 0.015625f : y) + ((r << 4) + 8u);
    int code = (int)(u >> 20) - (small ? 968 : 960);
    code = min(code, 126);
    if (mag > 0.0f) code = max(code, (int)least);
    if (!(mag < INFINITY)) code = 127;
    return (uint32_t)code;
}

template <typename T>
__device__ inline void read4(const T *p, int64_t at, int64_t n, bool whole, T (&x)[4])
{
    if (whole) {
        const vec4<T> q = *reinterpret_cast<const vec4<T> *>(p + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = q[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = at + e < n ? p[at + e] : (T)0;
    }
}
template <typename T>
__device__ inline void write4(T *p, int64_t at, int64_t n, bool whole, const T (&x)[4])
{
    if (whole) {
        vec4<T> q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = x[e];
        *reinterpret_cast<vec4<T> *>(p + at) = q;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) p[at + e] = x[e];
    }
}

template <typename P, typename G, bool MASTER, int BITS>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(AdamArgs a)
{
    using S = std::conditional_t<BITS == 8, uint8_t, float>;
    using W = std::conditional_t<MASTER, float, P>;
    int lo = 0, hi = a.n_tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const AdamTensor t = a.tensor[lo];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = (int64_t)(blockIdx.x - a.first[lo]) * kAdamChunk;
    P *const param = static_cast<P *>(t.param);
    const G *const grad = static_cast<const G *>(t.grad);
    W *const weight = MASTER ? reinterpret_cast<W *>(t.master) : reinterpret_cast<W *>(param);
    S *const ms = static_cast<S *>(t.m), *const vs = static_cast<S *>(t.v);
    // The factor of the gradients goes into these, which are rounded once: applied to every gradient it would be two roundings more of v.  Its power of
    // two is applied to the gradients, which is exact: the square of a factor of 1e-22, for gradients of 1e22, would be nothing.
    int power = 0;
    const double part = a.grad_scale ? (double)frexpf(*a.grad_scale, &power) : 1.0;
    const float in_m = (float)(a.one_less_beta1 * part), in_v = (float)(a.one_less_beta2 * part * part);

    W w[kAdamTurns][4];
    G g[kAdamTurns][4];
    S m8[kAdamTurns][4], v8[kAdamTurns][4];
    float m_scale[kAdamTurns], v_scale[kAdamTurns];
#pragma unroll
    for (int i = 0; i < kAdamTurns; ++i) {
        const int64_t block = chunk + (int64_t)(i * (kAdamThreads / 64) + wave) * kAdamBlock;
        if (block >= t.n) break;
        const int64_t at = block + 4 * lane;
        const bool whole = t.quads && at + 4 <= t.n;
        read4(weight, at, t.n, whole, w[i]);
        read4(grad, at, t.n, whole, g[i]);
        read4(ms, at, t.n, whole, m8[i]);
        read4(vs, at, t.n, whole, v8[i]);
        if constexpr (BITS == 8) {
            m_scale[i] = t.m_scale[block / kAdamBlock];
            v_scale[i] = t.v_scale[block / kAdamBlock];
        }
    }
#pragma unroll
    for (int i = 0; i < kAdamTurns; ++i) {
        const int64_t block = chunk + (int64_t)(i * (kAdamThreads / 64) + wave) * kAdamBlock;
        if (block >= t.n) break;
        const int64_t at = block + 4 * lane;
        const bool whole = t.quads && at + 4 <= t.n;
        float m[4], v[4], root[4];
        if constexpr (BITS == 8) {
            const uint32_t mw = m8[i][0] | m8[i][1] << 8 | m8[i][2] << 16 | (uint32_t)m8[i][3] << 24;
            const uint32_t vw = v8[i][0] | v8[i][1] << 8 | v8[i][2] << 16 | (uint32_t)v8[i][3] << 24;
            const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw, true);
            const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw, true);
            const float mc[4] = {m01[0], m01[1], m23[0], m23[1]}, vc[4] = {v01[0], v01[1], v23[0], v23[1]};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = mc[e] * m_scale[i];
                const float r = vc[e] * v_scale[i];
                v[e] = r * r;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { m[e] = m8[i][e]; v[e] = v8[i][e]; }
        }
        W out[4];
        P rounded[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = ldexpf((float)g[i][e], power);
            m[e] = m[e] * a.beta1 + ge * in_m;
            v[e] = v[e] * a.beta2 + (ge * in_v) * ge;
            root[e] = sqrtf(v[e]);
            const float p = (float)w[i][e] * a.keep - (m[e] / (root[e] * a.root + a.eps)) * a.step;
            out[e] = (W)p;
            rounded[e] = (P)p;
        }
        write4(weight, at, t.n, whole, out);
        if constexpr (MASTER) write4(param, at, t.n, whole, rounded);
        if constexpr (BITS == 8) {
            float m_most = 0.0f, v_most = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float am = fabsf(m[e]);
                if (at + e < t.n && am < INFINITY) m_most = fmaxf(m_most, am);
                if (at + e < t.n && root[e] < INFINITY) v_most = fmaxf(v_most, root[e]);
            }
            const int m_e = block_exponent(wave_max(m_most)), v_e = block_exponent(wave_max(v_most));
            const float m_inv = __uint_as_float((uint32_t)(127 - m_e) << 23), v_inv = __uint_as_float((uint32_t)(127 - v_e) << 23);
            S mo[4], vo[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint64_t r = mix(t.bits + kGamma * (uint64_t)(at / 2 + h + 1));
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int e = 2 * h + k;
                    const uint32_t r32 = k ? (uint32_t)(r >> 32) : (uint32_t)r;
                    mo[e] = (S)(encode(m[e], m_inv, r32 & 0xffffu, 0u) | (m[e] < 0.0f ? 128u : 0u));
                    vo[e] = (S)encode(root[e], v_inv, r32 >> 16, 1u);
                }
            }
            write4(ms, at, t.n, whole, mo);
            write4(vs, at, t.n, whole, vo);
            if (lane == 0) {
                t.m_scale[block / kAdamBlock] = __uint_as_float((uint32_t)(127 + m_e) << 23);
                t.v_scale[block / kAdamBlock] = __uint_as_float((uint32_t)(127 + v_e) << 23);
            }
        } else {
            write4(ms, at, t.n, whole, m);
            write4(vs, at, t.n, whole, v);
        }
    }
}

using AdamKernel = void (*)(AdamArgs);

template <int BITS>
AdamKernel adam_kernel(int32_t param, int32_t grad, bool master)
{
    if (param == RLS_F32) return adamw_kernel<float, float, false, BITS>;
    if (param == RLS_BF16) {
        if (grad == RLS_F32) return master ? adamw_kernel<__bf16, float, true, BITS> : adamw_kernel<__bf16, float, false, BITS>;
        return master ? adamw_kernel<__bf16, __bf16, true, BITS> : adamw_kernel<__bf16, __bf16, false, BITS>;
    }
    if (grad == RLS_F32) return master ? adamw_kernel<_Float16, float, true, BITS> : adamw_kernel<_Float16, float, false, BITS>;
    return master ? adamw_kernel<_Float16, _Float16, true, BITS> : adamw_kernel<_Float16, _Float16, false, BITS>;
}

int32_t check_tensor(const rls_adamw_tensor &t, int32_t state_bits)
{
    if (t.n < 0 || t.n > kAdamMost) return RLS_ERR_INVALID_ARG;
    if (!is_type(t.param_type) || (t.grad_type != RLS_F32 && t.grad_type != t.param_type)) return RLS_ERR_INVALID_ARG;
    if (t.n == 0) return RLS_OK;
    if (!t.param_dev || !t.grad_dev || !t.m_dev || !t.v_dev) return RLS_ERR_NULL;
    if (t.param_type == RLS_F32 && t.master_dev) return RLS_ERR_INVALID_ARG;
    if (state_bits == 8 && (!t.m_scale_dev || !t.v_scale_dev)) return RLS_ERR_NULL;
    return RLS_OK;
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" int32_t rls_adamw_step(const rls_adamw_tensor *tensors, int32_t n_tensors, const rls_adamw_options *options, void *stream)
{
    if (!options || (n_tensors > 0 && !tensors)) return RLS_ERR_NULL;
    const rls_adamw_options &o = *options;
    if (n_tensors < 0 || o.step < 1 || (o.state_bits != 32 && o.state_bits != 8)) return RLS_ERR_INVALID_ARG;
    if (!(o.beta1 >= 0.0 && o.beta1 < 1.0 && o.beta2 >= 0.0 && o.beta2 < 1.0)) return RLS_ERR_INVALID_ARG;
    if (!(isfinite(o.lr) && isfinite(o.weight_decay) && o.eps >= 0.0 && isfinite(o.eps))) return RLS_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const int32_t rc = check_tensor(tensors[i], o.state_bits);
        if (rc != RLS_OK) return rc;
    }
    AdamArgs a;
    a.beta1 = (float)o.beta1;
    a.one_less_beta1 = 1.0 - o.beta1;
    a.beta2 = (float)o.beta2;
    a.one_less_beta2 = 1.0 - o.beta2;
    a.keep = (float)(1.0 - o.lr * o.weight_decay);
    a.step = (float)(o.lr / (1.0 - pow(o.beta1, (double)o.step)));
    a.root = (float)(1.0 / sqrt(1.0 - pow(o.beta2, (double)o.step)));
    a.eps = (float)o.eps;
    a.grad_scale = o.grad_scale_dev;
    const uint64_t of_step = mix(o.seed + kGamma * (uint64_t)o.step);
    // kind by kind: the tensors of one go into launches of up to kTensors
    for (int kind = 0; kind < 18; ++kind) {
        const int32_t param = kind / 6, grad = kind % 2 ? RLS_F32 : param;
        const bool master = kind / 2 % 3 == 1;
        if (kind / 2 % 3 == 2 || (param == RLS_F32 && kind % 6 != 0)) continue;
        uint32_t blocks = 0;
        a.n_tensors = 0;
        auto launch = [&]() -> hipError_t {
            if (a.n_tensors == 0) return hipSuccess;
            const AdamKernel k = o.state_bits == 8 ? adam_kernel<8>(param, grad, master) : adam_kernel<32>(param, grad, master);
            hipLaunchKernelGGL(k, dim3(blocks), dim3(kAdamThreads), 0, (hipStream_t)stream, a);
            blocks = 0;
            a.n_tensors = 0;
            return hipGetLastError();
        };
        for (int32_t i = 0; i < n_tensors; ++i) {
            const rls_adamw_tensor &t = tensors[i];
            if (t.n == 0 || t.param_type != param || t.grad_type != grad || (t.master_dev != nullptr) != master) continue;
            const uint32_t nb = (uint32_t)((t.n + kAdamChunk - 1) / kAdamChunk);
            if (a.n_tensors == kTensors || blocks + nb > kAdamGrid) RLS_HIP_TRY(launch());
            const uintptr_t wide = (uintptr_t)t.master_dev | (param == RLS_F32 ? (uintptr_t)t.param_dev : 0) | (grad == RLS_F32 ? (uintptr_t)t.grad_dev : 0) |
                                   (o.state_bits == 32 ? (uintptr_t)t.m_dev | (uintptr_t)t.v_dev : 0);
            const uintptr_t half = (uintptr_t)t.param_dev | (uintptr_t)t.grad_dev;
            const uintptr_t bytes = (uintptr_t)t.m_dev | (uintptr_t)t.v_dev;
            const int32_t quads = wide % 16 == 0 && half % 8 == 0 && bytes % 4 == 0;
            a.tensor[a.n_tensors] = AdamTensor{t.param_dev, t.grad_dev, t.master_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev, t.n,
                                               mix(of_step + kGamma * (uint64_t)(i + 1)), quads};
            a.first[a.n_tensors++] = blocks;
            blocks += nb;
        }
        RLS_HIP_TRY(launch());
    }
    return RLS_OK;
}
