// The gated delta rule: a recurrence whose state is a matrix per head (rls.h gives the formulas), and its backward pass.
//
// Few steps are taken one by one, the state in registers: it is read and written once, which bounds it.
//
// Many are taken in chunks of 64.  With the sums of log-decays gamma inside a chunk, the state S0 before it, and over its steps i, j
//   a_i = exp(gamma_i), D_ij = exp(gamma_i - gamma_j) for j <= i, c_j = D_63,j, G = D . (K K^T) below the diagonal, P = D . (Q K^T),
// where what a reset lies between is 0, the differences y_i = v_i - (decayed state)^T k_i of all steps are one triangular system,
//   (1 + G beta) Y = V - a . (K S0),  so with X = (1 + G beta)^-1   Y = X (V - a . (K S0)),  S1 = a_63 S0 + (c beta K)^T Y,
//   O = scale (a . (Q S0) + P (beta Y)).
// X and P are made for all chunks at once; then a chain of these products per chunk runs for 16 columns of the state at a time, with the outputs in it.
// The backward pass keeps S0 and Y of every chunk, has a chain from the last chunk to the first,
//   dY = X^T beta (scale P^T dO + c . (K dS1)),  dS0 = a_63 dS1 + scale (a Q)^T dO - (a K)^T dY,
// and then takes all other gradients at once.
// The state is handed back in fp32, and what it is made of must not be rounded to fewer bits on the way.  So a matrix instruction of 16-bit operands takes an
// fp32 number as the sum of three bf16 numbers (24 bits, what is left out is 2^-27 of it), an fp16 input as two and a bf16 input as it is, and of the products
// of two such sums those that count in fp32: three for a bf16 input with an fp32 operand, six for two of fp32, at 1/16 of an fp32 instruction's time each.
// Small and awkward products (the inverse) are left to the fp32 instructions.
// What it takes, heads of 128 x 128 in bf16: a token of 64 x 32 heads 59 us (4.6 TB/s of state); 8191 steps of 32 heads 361 a pass, in a profiler's trace 2 x 57 to
// prepare the chunks and 2 x 136 in the chain, 2.1 a chunk (all of it with fp32 instructions and outputs apart: 1349); gradients of 4 x 2048 steps of 16
// heads 610 a pass, in a trace 77, 151, 190 in the chain back, 202 for all gradients (1288).  fp16 and fp32: 8191 steps 547 and 716, gradients 864 and 1040.
#include <algorithm>
#include <type_traits>

#include "element_types.h"
#include "rls_internal.h"
#include "wave.h"

namespace rls {

namespace {

constexpr int kChunk = 64;
constexpr int kEdge = kChunk + 4;                        // row of a chunk x chunk matrix in LDS (4 modulo 16: no bank is asked twice, by rows or by columns)
constexpr float kNoCarry = -87.0f;                       // exp of less is below the smallest normal number

using f4 = vec4<float>;

struct Heads {
    void *data;
    int64_t batch, step, head;                           // distances in elements
};
struct DeltaArgs {
    Heads q, k, v, o, dout, dq, dk, dv;
    const float *g, *beta;                               // [batch][steps][heads]
    const uint8_t *reset;                                // [batch][steps]
    const float *state;                                  // before the first chunk of the launch, [batch * heads][dk][dv], or null
    float *last;                                         // after the last one
    float *dg, *dbeta;
    int64_t batch, steps, chunk0;                        // the launch takes chunks chunk0 .. chunk0 + chunks - 1
    int32_t heads, group, chunks;                        // group: heads that share a key head
    int32_t key_dim, value_dim, columns, slices;         // columns: value_dim rounded up to 64; slices: of 16 columns, that a chain goes through
    float scale;
    // workspace, an entry per (head, chunk of the launch)
    float *y, *s, *dy, *ds, *gq, *gk;                    // [64][columns], [DK][columns], the same two, [64][DK] x 2
    float *carry;                                        // a_63
    float *gates;                                        // [2][64]: a, c beta
    float *spare;                                        // 64 numbers that nothing reads
    // planes, in the order in which the chain's lanes hold them: of X and scale P beta (backward: turned, and X^T beside X); per (key head, chunk) of
    // K, Q, K^T (and Q^T)
    __bf16 *xp, *pp, *xt, *kp, *qp, *kt, *qt;
    int32_t keep;                                        // for the backward pass
};

// A kernel's arguments read anew, for code behind its loops that hardly any call reaches: none of them is kept in a register until then
__device__ inline const DeltaArgs &arguments_again()
{
    auto *const held = __builtin_amdgcn_kernarg_segment_ptr();
    uint64_t at = (uint64_t)held;
    asm volatile("" : "+s"(at));
    return *(const DeltaArgs *)at;
}

template <typename T>
__device__ inline const T *at(const Heads &h, int64_t b, int64_t t, int64_t head)
{
    return static_cast<const T *>(h.data) + b * h.batch + t * h.step + head * h.head;
}
template <typename T>
__device__ inline T *out_at(const Heads &h, int64_t b, int64_t t, int64_t head)
{
    return static_cast<T *>(h.data) + b * h.batch + t * h.step + head * h.head;
}

// ---- matrix instructions ----------------------------------------------------------------------------------------------
// An operand of 16 x 16 x 16: lane l has four numbers along the axis that is summed over, from 4 (l / 16) on, of row (or column) l % 16.  A result
// has the same form with its rows in the place of that axis, so it can be the next product's right operand as it is.

__device__ inline int lane16() { return threadIdx.x & 15; }
__device__ inline int lane4() { return (threadIdx.x & 63) >> 4 << 2; }

__device__ inline f4 mm(f4 a, f4 b, f4 c)
{
#pragma unroll
    for (int m = 0; m < 4; ++m) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[m], b[m], c, 0, 0, 0);
    return c;
}
// the summed axis along the rows of memory
__device__ inline f4 along(const float *p, int ld, int row, int k)
{
    return *reinterpret_cast<const f4 *>(p + (row + lane16()) * ld + k + lane4());
}
// and across them
__device__ inline f4 across(const float *p, int ld, int k, int column)
{
    const float *const q = p + (k + lane4()) * ld + column + lane16();
    return f4{q[0], q[ld], q[2 * ld], q[3 * ld]};
}
__device__ inline void put(float *p, int ld, int row, int column, f4 v)
{
    float *const q = p + (row + lane4()) * ld + column + lane16();
#pragma unroll
    for (int m = 0; m < 4; ++m) q[m * ld] = v[m];
}
__device__ inline f4 four(const float *p, int k) { return *reinterpret_cast<const f4 *>(p + k + lane4()); }

// ---- numbers as sums of bf16 numbers -----------------------------------------------------------------------------------
// An operand of 16 x 16 x 32: lane l has eight numbers along the axis that is summed over, from 8 (l / 16) on, of row (or column) l % 16.

using b8 = vec8<__bf16>;
using b4 = vec4<__bf16>;

template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : std::is_same<T, __bf16>::value ? 1 : 2;

template <int N, typename B, typename F>
__device__ inline void split(F x, B (&to)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        to[i] = __builtin_convertvector(x, B);
        x -= __builtin_convertvector(to[i], F);
    }
}
template <typename T>
struct Raw {                                             // eight inputs as they come
    T x[8];
};
template <typename T, int N>
__device__ inline void planes_of(const Raw<T> &r, b8 (&to)[N])
{
    vec8<float> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)r.x[i];
    split(x, to);
}
template <>
__device__ inline void planes_of<__bf16, 1>(const Raw<__bf16> &r, b8 (&to)[1])
{
    __builtin_memcpy(&to[0], r.x, 16);
}
// eight inputs of a row from column d on, 0 where there are none
template <typename T>
__device__ inline Raw<T> load_raw(const T *row, bool in, int d, int columns)
{
    Raw<T> r;
    if (in && d + 8 <= columns) {
        __builtin_memcpy(r.x, row + d, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.x[i] = in && d + i < columns ? row[d + i] : (T)0.0f;
    }
    return r;
}
template <int NA, int NB>
__device__ inline f4 mmp(const b8 (&a)[NA], const b8 (&b)[NB], f4 c)
{
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i + j == sum) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c, 0, 0, 0);
    return c;
}
// Memory in the order of the lanes: a block of 64 x 8 numbers for every 16 rows, 32 of the summed axis and plane.  Where number k (a multiple of 8) of a
// row begins, with `blocks` blocks along the summed axis and N planes
template <int N>
__device__ inline int place_in(int row, int k, int blocks, int plane)
{
    return (((row >> 4) * blocks + (k >> 5)) * N + plane) * 512 + ((row & 15) + ((k & 31) >> 3) * 16) * 8;
}
template <int N>
__device__ inline void load_block(b8 (&to)[N], const __bf16 *p, int block)
{
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = *reinterpret_cast<const b8 *>(p + (block * N + i) * 512 + (threadIdx.x & 63) * 8);
}
// two chains of products, none waits for more than half of the others
template <int NA, int NB>
__device__ inline void mmp(const b8 (&a)[NA], const b8 (&b)[NB], f4 &even, f4 &odd)
{
    int n = 0;
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i + j == sum) {
                    f4 &c = n++ & 1 ? odd : even;
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c, 0, 0, 0);
                }
}
__device__ inline int lane8() { return (threadIdx.x & 63) >> 4 << 3; }
// from planes in memory, rows ld apart and planes `plane` apart
template <int N>
__device__ inline void load_planes(b8 (&to)[N], const __bf16 *p, int plane, int ld, int row, int k)
{
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = *reinterpret_cast<const b8 *>(p + i * plane + (row + lane16()) * ld + k + lane8());
}
// a result (four rows, from `row` on, of 16 columns) as the next product's right operand, which sums over the rows: blocks in the order of the lanes, so that no
// bank is asked twice
template <int N = 3>
__device__ inline void put_block(__bf16 *p, int row, f4 v)
{
    b4 to[N];
    split(v, to);
    const int k = row + lane4();
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<b4 *>(p + place_in<N>(lane16(), k, 1, i) + (k & 4)) = to[i];
}

// The tiles on and below the diagonal of a chunk x chunk matrix
constexpr int kLower = 10;
__device__ inline void lower_tile(int u, int &ti, int &tj)
{
    ti = u < 1 ? 0 : u < 3 ? 1 : u < 6 ? 2 : 3;
    tj = u - ti * (ti + 1) / 2;
}

// ---- the gates of a chunk ----------------------------------------------------------------------------------------------

struct alignas(16) Gates {
    double gamma[kChunk];                                // times log2(e)
    float beta[kChunk], a[kChunk], c[kChunk];
    int32_t part[kChunk];                                // resets up to here
    uint8_t cut[kChunk];

    // by the first wave; the others see it after a barrier
    __device__ void load(const DeltaArgs &p, int64_t b, int64_t head, int64_t t0)
    {
        const int l = threadIdx.x;
        if (l >= kChunk) return;
        const int64_t t = min(t0 + l, p.steps - 1), i = (b * p.steps + t) * p.heads + head;
        const bool in = t0 + l < p.steps;
        const float g = p.g[i], given = p.beta[i];
        const uint8_t reset = p.reset ? p.reset[b * p.steps + t] : 0;
        const bool no_carry = in && (g < kNoCarry || reset != 0);
        beta[l] = in ? given : 0.0f;
        cut[l] = no_carry;
        const double sum = wave_scan(!in || no_carry ? 0.0 : (double)g * 1.4426950408889634, 0.0, [](double x, double y) { return x + y; });
        const uint64_t cuts = __ballot(no_carry);
        const int before = __popcll(cuts & (l == 63 ? ~0ull : (1ull << (l + 1)) - 1));
        gamma[l] = sum;
        part[l] = before;
        a[l] = before == 0 ? __builtin_amdgcn_exp2f((float)sum) : 0.0f;
        const double end = last_lane(sum);
        c[l] = before == __popcll(cuts) ? __builtin_amdgcn_exp2f((float)(end - sum)) : 0.0f;
    }
    // The sums anew, each from a cut on, for gates that are not finite: those do not go away by being subtracted
    __device__ void sum_within_cuts(const DeltaArgs &p, int64_t gate, int l, bool in)
    {
        double sum = in && !cut[l] ? (double)p.g[gate] * 1.4426950408889634 : 0.0;
        for (int step = 1; step < kChunk; step <<= 1) {
            const double before = __shfl_up(sum, step);
            if (l >= step && part[l - step] == part[l]) sum += before;
        }
        const double end = __shfl(sum, kChunk - 1);
        gamma[l] = sum;
        a[l] = part[l] == 0 ? __builtin_amdgcn_exp2f((float)sum) : 0.0f;
        c[l] = part[l] == part[kChunk - 1] ? __builtin_amdgcn_exp2f((float)(end - sum)) : 0.0f;
    }
    __device__ float decay(int i, int j) const { return j <= i && part[i] == part[j] ? __builtin_amdgcn_exp2f((float)(gamma[i] - gamma[j])) : 0.0f; }
};

// ---- all chunks at once: X, P and K^T -------------------------------------------------------------------------------------

template <typename T, int DK>
__global__ void __launch_bounds__(256) delta_prepare_kernel(DeltaArgs p)
{
    constexpr int NI = kPlanes<T>, LD = DK + 8, Plane = kChunk * LD;
    __shared__ Gates gates;
    constexpr int XBytes = kChunk * kEdge * 4, QBytes = NI * Plane * 2;
    __shared__ __attribute__((aligned(16))) __bf16 k[NI * Plane];
    __shared__ __attribute__((aligned(16))) char qx[QBytes > XBytes ? QBytes : XBytes];
    __bf16 *const q = reinterpret_cast<__bf16 *>(qx);
    float *const x = reinterpret_cast<float *>(qx);      // X comes when q has been used
    __shared__ __attribute__((aligned(16))) float n[kChunk * kEdge];             // G beta below the diagonal; scale P beta, turned, from it on
    const int wave = threadIdx.x >> 6;
    const int64_t unit = blockIdx.x, bh = unit / p.chunks, chunk = unit % p.chunks, b = bh / p.heads, head = bh % p.heads, key = head / p.group;
    const int64_t t0 = (p.chunk0 + chunk) * kChunk, inputs = ((b * (p.heads / p.group) + key) * p.chunks + chunk) * NI * kChunk * DK;
    const bool first = head % p.group == 0;              // of the heads that share the keys: it writes their planes
    // (a wave reads what makes one block, so that it writes a kilobyte in a row)
    const int in_block = threadIdx.x & 15, along_block = (threadIdx.x & 63) >> 4 << 3;
    Raw<T> raw_k[DK / 32], raw_q[DK / 32];               // (all asked for before the first is used)
#pragma unroll
    for (int e = 0; e < DK / 32; ++e) {
        const int u = wave + 4 * e, row = u / (DK / 32) * 16 + in_block, d = u % (DK / 32) * 32 + along_block;
        const bool in = t0 + row < p.steps;
        raw_k[e] = load_raw(at<T>(p.k, b, t0 + row, key), in, d, p.key_dim);
        raw_q[e] = load_raw(at<T>(p.q, b, t0 + row, key), in, d, p.key_dim);
    }
    gates.load(p, b, head, t0);
#pragma unroll
    for (int e = 0; e < DK / 32; ++e) {
        const int u = wave + 4 * e, row = u / (DK / 32) * 16 + in_block, d = u % (DK / 32) * 32 + along_block;
        b8 pk[NI], pq[NI];
        planes_of(raw_k[e], pk);
        planes_of(raw_q[e], pq);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            *reinterpret_cast<b8 *>(k + i * Plane + row * LD + d) = pk[i];
            *reinterpret_cast<b8 *>(q + i * Plane + row * LD + d) = pq[i];
            if (first) {
                *reinterpret_cast<b8 *>(p.kp + inputs + place_in<NI>(row, d, DK / 32, i)) = pk[i];
                *reinterpret_cast<b8 *>(p.qp + inputs + place_in<NI>(row, d, DK / 32, i)) = pq[i];
            }
        }
    }
    __syncthreads();
    for (int u = wave; u < kLower; u += 4) {
        int ti, tj;
        lower_tile(u, ti, tj);
        f4 kk{}, qk{};
#pragma unroll
        for (int kb = 0; kb < DK; kb += 32) {
            b8 left[NI], right[NI];
            load_planes(right, k, Plane, LD, tj * 16, kb);
            load_planes(left, k, Plane, LD, ti * 16, kb);
            kk = mmp(left, right, kk);
            load_planes(left, q, Plane, LD, ti * 16, kb);
            qk = mmp(left, right, qk);
        }
        const int j = tj * 16 + lane16();
        const float beta = gates.beta[j];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int i = ti * 16 + lane4() + m;
            const float decay = gates.decay(i, j) * beta;
            if (j < i) n[i * kEdge + j] = kk[m] * decay;
            if (j <= i) n[j * kEdge + i] = qk[m] * decay * p.scale;
        }
    }
    if (first) {
        for (int u = wave; u < DK / 16 * 2; u += 4) {
            const int d = u / 2 * 16 + in_block, t = u % 2 * 32 + along_block;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                b8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k[i * Plane + (t + e) * LD + d];
                *reinterpret_cast<b8 *>(p.kt + inputs + place_in<NI>(d, t, 2, i)) = v;
                if (!p.keep) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = q[i * Plane + (t + e) * LD + d];
                *reinterpret_cast<b8 *>(p.qt + inputs + place_in<NI>(d, t, 2, i)) = v;
            }
        }
    }
    __syncthreads();
    // blocks on the diagonal: a lane solves for a column
    if ((threadIdx.x & 63) < 16) {
        const int column = threadIdx.x & 63;
        const float *const nd = n + wave * 16 * kEdge + wave * 16;
        float col[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = column == i ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j) sum = fmaf(-nd[i * kEdge + j], col[j], sum);
            col[i] = sum;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(wave * 16 + i) * kEdge + wave * 16 + column] = col[i];
    }
    __syncthreads();
    // block (i, j) = -X_ii (sum over j <= l < i of N_il X_lj), one diagonal after the other
    for (int apart = 1; apart < 4; ++apart) {
        if (wave + apart < 4) {
            const int j = wave, i = j + apart;
            f4 sum{};
            for (int l = j; l < i; ++l) sum = mm(along(n, kEdge, i * 16, l * 16), across(x, kEdge, l * 16, j * 16), sum);
            put(x, kEdge, i * 16, j * 16, -mm(along(x, kEdge, i * 16, i * 16), sum, f4{}));
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) p.carry[unit] = gates.a[kChunk - 1];
    if (threadIdx.x < kChunk) {
        float *const to = p.gates + unit * 2 * kChunk + threadIdx.x;
        to[0] = gates.a[threadIdx.x];
        to[kChunk] = gates.c[threadIdx.x] * gates.beta[threadIdx.x];
    }
    for (int u = wave; u < 8; u += 4) {
        const int i = u / 2 * 16 + in_block, j = u % 2 * 32 + along_block;
        vec8<float> vx, vp, vt;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            vx[e] = j + e <= i ? x[i * kEdge + j + e] : 0.0f;
            if (p.keep) {
                vp[e] = j + e >= i ? n[i * kEdge + j + e] : 0.0f;
                vt[e] = j + e >= i ? x[(j + e) * kEdge + i] : 0.0f;
            } else {
                vp[e] = j + e <= i ? n[(j + e) * kEdge + i] : 0.0f;
            }
        }
        b8 px[3], pp[3], pt[3];
        split(vx, px);
        split(vp, pp);
        if (p.keep) split(vt, pt);
#pragma unroll
        for (int plane = 0; plane < 3; ++plane) {
            const int64_t to = unit * 3 * kChunk * kChunk + place_in<3>(i, j, 2, plane);
            *reinterpret_cast<b8 *>(p.xp + to) = px[plane];
            *reinterpret_cast<b8 *>(p.pp + to) = pp[plane];
            if (p.keep) *reinterpret_cast<b8 *>(p.xt + to) = pt[plane];
        }
    }
}

// ---- the chain over chunks, 16 columns of the state by a workgroup --------------------------------------------------------
// Eight waves, 16 of the chunk's steps for two of them.  The first four: R = V - a (K S), Y = X R.  The other four, beside them: o = scale a (Q S)
// + scale P beta Y, a chunk's last product beside the next chunk's first, and what can be done ahead (V) or later (Y's planes) for the first four.
// Then all of them: S = carry S + K^T (c beta Y), 16 rows of it each.  Three barriers a chunk; what a chunk needs of memory is read while the one before
// it is worked on.  The first four's path bounds it: splits of numbers, LDS and the latency of some 30 matrix instructions.

// rows (operands of 32 numbers of the summed axis each) times planes in LDS, which are asked for two blocks ahead of their products
template <int NI, int BLOCKS>
__device__ inline f4 rows_by(const b8 (&rows)[BLOCKS][NI], const __bf16 *planes)
{
    b8 s[2][3];
    load_block(s[0], planes, 0);
    if (BLOCKS > 1) load_block(s[1], planes, 1);
    __builtin_amdgcn_sched_barrier(0);
    f4 c[4] = {};
#pragma unroll
    for (int kb = 0; kb < BLOCKS; ++kb) {
        mmp(rows[kb], s[kb & 1], c[kb & 1 ? 2 : 0], c[kb & 1 ? 3 : 1]);
        if (kb + 2 < BLOCKS) load_block(s[kb & 1], planes, kb + 2);
        __builtin_amdgcn_sched_barrier(0);
    }
    return (c[0] + c[1]) + (c[2] + c[3]);
}

// Every wave of a kind has the same loads and stores in the same order, none of them behind a branch, so that it waits for a load by how many came after it
// and for nothing else: what has no place to go is stored to a spare one.  Products with a block of zeros are taken too, for the same reason and because
// the compiler has left out the wait states between a matrix instruction and what read its result behind a branch to an earlier block (a test looks for that
// along every path of the listings).
// Steps behind the last one are worked on with the last one's v: beta is 0 there, and what they give is not written.
template <int DK>
struct alignas(16) ChainShared {
    __bf16 s[3 * 16 * DK], r[3 * 16 * kChunk], y[3 * 16 * kChunk], u[3 * 16 * kChunk];
    f4 v[4][64], y32[4][64];                             // as lanes hold them
};
// Four rows of a chunk (from `row` on) of an array of heads: how far they are from the chunk's first row.  A chunk's last rows may lie behind the last step;
// they are read as the last step's.
struct Rows {
    int64_t apart[4];
    __device__ void set(int row, int64_t step, int64_t steps)                    // steps: from the chunk's first row on
    {
        const int most = (int)min<int64_t>(kChunk, steps) - 1;
#pragma unroll
        for (int m = 0; m < 4; ++m) apart[m] = min(row + m, most) * step;
    }
};
__device__ inline void all_waves()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ inline bool not_finite(f4 state)
{
    bool bad = false;
#pragma unroll
    for (int m = 0; m < 4; ++m) bad |= !(fabsf(state[m]) < INFINITY);
    return bad;
}
// 16 rows and columns of the state at the end, column j by this lane
__device__ inline void put_state(const DeltaArgs &p, int64_t bh, int row, int j, f4 state)
{
    if (!p.last || j >= p.value_dim) return;
#pragma unroll
    for (int m = 0; m < 4; ++m)
        if (row + lane4() + m < p.key_dim) p.last[(bh * p.key_dim + row + lane4() + m) * p.value_dim + j] = state[m];
}

// Returns the state at the end, 16 rows of a wave
template <typename T, int DK, bool KEEP, bool ANSWERS>
__device__ inline f4 run_chain(const DeltaArgs &p, ChainShared<DK> &sh, int64_t bh, int slice)
{
    constexpr int NI = kPlanes<T>, Square = kChunk * kChunk, Inputs = NI * kChunk * DK;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tile = wave & 3;
    const bool mine = wave < DK / 16;                    // it has 16 rows of the state
    const int64_t b = bh / p.heads, head = bh % p.heads, key = head / p.group, kbh = b * (p.heads / p.group) + key;
    const int column = slice * 16, j = column + lane16();
    f4 state{};
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int row = wave * 16 + lane4() + m;
        if (p.state && mine && row < p.key_dim && j < p.value_dim) state[m] = p.state[(bh * p.key_dim + row) * p.value_dim + j];
    }
    // where a wave's part of a chunk begins; the next chunk's follows behind it
    const __bf16 *rows_at = (ANSWERS ? p.qp : p.kp) + kbh * p.chunks * Inputs + tile * (DK / 32) * NI * 512;
    const __bf16 *left_at = (ANSWERS ? p.pp : p.xp) + bh * p.chunks * 3 * Square + tile * 2 * 3 * 512;
    const __bf16 *kt_at = p.kt + kbh * p.chunks * Inputs + (mine ? wave : 0) * 2 * NI * 512;
    const float *a_at = p.gates + bh * p.chunks * 2 * kChunk + tile * 16, *cbeta_at = a_at + kChunk, *carry_at = p.carry + bh * p.chunks;
    const int row = tile * 16 + lane4(), steps_left = (int)min<int64_t>(p.steps - p.chunk0 * kChunk, (int64_t)p.chunks * kChunk);   // of this launch
    const T *v_at = at<T>(p.v, b, p.chunk0 * kChunk, head) + min(j, p.value_dim - 1);
    T *o_at = KEEP ? nullptr : out_at<T>(p.o, b, p.chunk0 * kChunk + row, head) + j, *const spare = reinterpret_cast<T *>(p.spare) + (threadIdx.x & 63);
    constexpr bool kQueries = ANSWERS && !KEEP;          // for the backward pass nothing is answered
    b8 rows[DK / 32][NI], left[2][3], kt[2][NI];
    T v[4];
    f4 a, cbeta{}, by_query{};
    float carry;
    // a chunk's loads in groups, each right after the last use of what it takes the place of
    const auto load_rows_of = [&]() {
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) load_block(rows[kb], rows_at, kb);
        a = four(a_at, 0);
    };
    const auto load_left_of = [&]() {
        load_block(left[0], left_at, 0);
        load_block(left[1], left_at, 1);
        if (!ANSWERS) cbeta = four(cbeta_at, 0);
    };
    const auto load_kt_of = [&]() {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) load_block(kt[kb], kt_at, kb);
        carry = *carry_at;
    };
    // (chunk after chunk)
    const auto load_v_of = [&](int n) {
        const int most = min(kChunk, steps_left - n * kChunk) - 1;
#pragma unroll
        for (int m = 0; m < 4; ++m) v[m] = v_at[min(row + m, most) * p.v.step];
        if (n + 1 < p.chunks) v_at += kChunk * p.v.step;
    };
    const auto put_v = [&]() { sh.v[tile][threadIdx.x & 63] = f4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}; };
    // + scale P beta Y, of chunk n
    const auto answer = [&](int n) {
        f4 o = by_query * p.scale;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            b8 y[3];
            load_block(y, sh.y, kb);
            o = mmp(left[kb], y, o);
            __builtin_amdgcn_sched_barrier(0);
        }
        const int rows_in = j < p.value_dim ? steps_left - n * kChunk - row : 0;
#pragma unroll
        for (int m = 0; m < 4; ++m) *(m < rows_in ? o_at + m * p.o.step : spare) = (T)o[m];
        o_at += kChunk * p.o.step;
    };
    if (!ANSWERS) __builtin_amdgcn_s_setprio(3);         // the others wait for them
    if (!ANSWERS || kQueries) {
        load_rows_of();
        load_left_of();
    }
    if (ANSWERS) {
        load_v_of(0);
        put_v();
        load_v_of(min(1, p.chunks - 1));
    }
    load_kt_of();
    for (int n = 0; n < p.chunks; ++n) {
        const int64_t unit = bh * p.chunks + n;
        if (n + 1 < p.chunks) {                          // (behind the last chunk the loads are of the last one again)
            rows_at += Inputs;
            kt_at += Inputs;
            a_at += 2 * kChunk;
            cbeta_at += 2 * kChunk;
            ++carry_at;
        }
        if (ANSWERS ? n > 0 : n + 1 < p.chunks) left_at += 3 * Square;         // (P is needed a chunk later)
        if (mine) {
            put_block(sh.s, wave * 16, state);
            if (KEEP) put(p.s + unit * DK * p.columns, p.columns, wave * 16, column, state);
        }
        all_waves();
        if (!ANSWERS) {
            const f4 x = sh.v[tile][threadIdx.x & 63];
            put_block(sh.r, tile * 16, x - rows_by(rows, sh.s) * a);
            load_rows_of();
        } else if (kQueries && n > 0) {
            answer(n - 1);
            load_left_of();
        }
        all_waves();
        if (!ANSWERS) {
            b8 r[2][3];
            load_block(r[0], sh.r, 0);
            load_block(r[1], sh.r, 1);
            __builtin_amdgcn_sched_barrier(0);
            f4 c[4] = {};
            mmp(left[0], r[0], c[0], c[1]);
            mmp(left[1], r[1], c[2], c[3]);
            const f4 y = (c[0] + c[1]) + (c[2] + c[3]);
            put_block(sh.u, tile * 16, y * cbeta);
            if (KEEP) put(p.y + unit * kChunk * p.columns, p.columns, tile * 16, column, y);
            else sh.y32[tile][threadIdx.x & 63] = y;
            load_left_of();
        } else {
            put_v();
            load_v_of(min(n + 2, p.chunks - 1));
            if (kQueries) {
                // (a state may be finite and its product with a query not: behind a cut neither counts, and nothing of it is left in the state to tell)
                by_query = rows_by(rows, sh.s);
#pragma unroll
                for (int m = 0; m < 4; ++m) by_query[m] = a[m] == 0.0f ? 0.0f : by_query[m] * a[m];
                load_rows_of();
            }
        }
        all_waves();
        b8 u[2][3];
        load_block(u[0], sh.u, 0);
        load_block(u[1], sh.u, 1);
        __builtin_amdgcn_sched_barrier(0);
        f4 c[4] = {state * carry, f4{}, f4{}, f4{}};
        mmp(kt[0], u[0], c[0], c[1]);
        mmp(kt[1], u[1], c[2], c[3]);
        state = (c[0] + c[1]) + (c[2] + c[3]);
        if (kQueries) put_block(sh.y, tile * 16, sh.y32[tile][threadIdx.x & 63]);
        load_kt_of();
    }
    all_waves();
    if (kQueries) answer(p.chunks - 1);                  // (the four of them by themselves: each reads what all of them have put)
    return state;
}

// What a chain multiplies by 0 - the state before a reset, steps on the other side of one - does not go away if it is infinite or no number.  Once in the state
// it stays there to the chain's end, so the state that is left tells: a workgroup whose columns are not finite then takes them again, step by step, where
// a cut is no product.  A column has 32 lanes.  (1.2 to 4 us a step, for calls that hold such numbers only.)
__device__ inline float column_sum(float x)              // over 32 lanes
{
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// a column of the state, every 32nd row a lane
template <int DK>
struct Column {
    static constexpr int R = DK / 32;
    float s[R];
    int64_t place;                                       // of its first row, in p.state and p.last
    int j;
    bool in;

    int lane;                                            // of 32
    __device__ int row(int i) const { return lane + 32 * i; }
    __device__ Column(const DeltaArgs &p, int64_t bh, int slice) : j(slice * 16 + (int)(threadIdx.x >> 5)), lane(threadIdx.x & 31)
    {
        in = j < p.value_dim;
        place = bh * p.key_dim * p.value_dim + j;
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = p.state && in && row(i) < p.key_dim ? p.state[place + (int64_t)row(i) * p.value_dim] : 0.0f;
    }
    __device__ void put_last(const DeltaArgs &p) const
    {
        if (!p.last || !in) return;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row(i) < p.key_dim) p.last[place + (int64_t)row(i) * p.value_dim] = s[i];
    }
    __device__ void keep(float *to, int columns) const   // with zeros where the state has no rows and columns
    {
#pragma unroll
        for (int i = 0; i < R; ++i) to[row(i) * columns + j] = in ? s[i] : 0.0f;
    }
};
template <typename T, int DK, bool KEEP>
__device__ void chain_by_steps(const DeltaArgs &p, int64_t bh, int slice)
{
    const int64_t b = bh / p.heads, head = bh % p.heads, key = head / p.group;
    Column<DK> c(p, bh, slice);
#pragma unroll 1
    for (int n = 0; n < p.chunks; ++n) {
        const int64_t unit = bh * p.chunks + n, t0 = (p.chunk0 + n) * kChunk;
        if (KEEP) c.keep(p.s + unit * DK * p.columns, p.columns);
#pragma unroll 1
        for (int l = 0; l < kChunk; ++l) {
            const int64_t t = t0 + l, gate = (b * p.steps + t) * p.heads + head;
            float y = 0.0f;
            if (t < p.steps) {
                const T *const k = at<T>(p.k, b, t, key), *const q = at<T>(p.q, b, t, key);
                const bool cut = p.g[gate] < kNoCarry || (p.reset && p.reset[b * p.steps + t] != 0);
                const float carry = cut ? 0.0f : expf(p.g[gate]);
                float sk = 0.0f, sq = 0.0f;
#pragma unroll
                for (int i = 0; i < c.R; ++i) {
                    c.s[i] = cut ? 0.0f : c.s[i] * carry;
                    if (c.row(i) < p.key_dim) sk = fmaf(c.s[i], (float)k[c.row(i)], sk);
                }
                y = c.in ? (float)at<T>(p.v, b, t, head)[c.j] - column_sum(sk) : 0.0f;
                const float u = p.beta[gate] * y;
#pragma unroll
                for (int i = 0; i < c.R; ++i)
                    if (c.row(i) < p.key_dim) {
                        c.s[i] = fmaf((float)k[c.row(i)], u, c.s[i]);
                        sq = fmaf(c.s[i], (float)q[c.row(i)], sq);
                    }
                if (!KEEP) {
                    const float o = p.scale * column_sum(sq);
                    if (c.in && c.lane == 0) out_at<T>(p.o, b, t, head)[c.j] = (T)o;
                }
            }
            if (KEEP && c.lane == 0) p.y[(unit * kChunk + l) * p.columns + c.j] = y;
        }
    }
    c.put_last(p);
}

template <typename T, int DK, bool KEEP>
__global__ void __launch_bounds__(512, kPlanes<T> == 1 ? 4 : 2) delta_chain_kernel(DeltaArgs p)
{
    __shared__ ChainShared<DK> sh;
    __shared__ int32_t bad;
    if (threadIdx.x == 0) bad = 0;
    // workgroups go round the 8 dies in turn; those of a head read the same matrices and share a die's cache
    const int64_t die = blockIdx.x & 7, place = blockIdx.x >> 3, bh = place / p.slices * 8 + die;
    if (bh >= p.batch * p.heads) return;
    const int slice = (int)(place % p.slices);
    const f4 state = threadIdx.x < 256 ? run_chain<T, DK, KEEP, false>(p, sh, bh, slice) : run_chain<T, DK, KEEP, true>(p, sh, bh, slice);
    const int wave = threadIdx.x >> 6;
    if (wave < DK / 16 && not_finite(state)) bad = 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(bad)) chain_by_steps<T, DK, KEEP>(arguments_again(), bh, slice);
    else if (wave < DK / 16) put_state(p, bh, wave * 16, slice * 16 + lane16(), state);
}

// ---- backward: the chain from the last chunk to the first ----------------------------------------------------------------
// Z = c beta (K dS) + E and dY = X^T Z by the first four waves, then by all of them dS = carry dS + Q^T (scale a dO) - K^T (a dY).  The other four are a
// chunk ahead with what depends on dO alone: E = (scale P beta)^T dO, and scale a dO.  dS behind every chunk goes to ds, dY to dy.  Loads and stores as in
// the forward chain.

template <typename T, int DK>
struct alignas(16) BackShared {
    // (q is read to a chunk's end, so the next chunk's has a place of its own)
    __bf16 s[3 * 16 * DK], o[kPlanes<T> * 16 * kChunk], q[2][3 * 16 * kChunk], z[3 * 16 * kChunk], u[3 * 16 * kChunk];
    f4 e[4][64];
    int32_t bad;                                         // the state at the end is not finite
};

// Returns whether the state at the end is finite; if not, it is not written
template <typename T, int DK, bool FEEDS>
__device__ inline bool run_back_chain(const DeltaArgs &p, BackShared<T, DK> &sh, int64_t bh, int slice)
{
    constexpr int NI = kPlanes<T>, Square = kChunk * kChunk, Inputs = NI * kChunk * DK;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tile = wave & 3;
    const bool mine = wave < DK / 16;
    const int64_t b = bh / p.heads, head = bh % p.heads, key = head / p.group, kbh = b * (p.heads / p.group) + key, end = p.chunks - 1;
    const int column = slice * 16, j = column + lane16();
    if (threadIdx.x == 0) sh.bad = 0;
    f4 state{};
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int row = wave * 16 + lane4() + m;
        if (p.state && mine && row < p.key_dim && j < p.value_dim) state[m] = p.state[(bh * p.key_dim + row) * p.value_dim + j];
    }
    const __bf16 *rows_at = p.kp + (kbh * p.chunks + end) * Inputs + tile * (DK / 32) * NI * 512;
    const __bf16 *square_at = (FEEDS ? p.pp : p.xt) + (bh * p.chunks + end) * 3 * Square + tile * 2 * 3 * 512;
    const int64_t turned = (kbh * p.chunks + end) * Inputs + (mine ? wave : 0) * 2 * NI * 512;
    const __bf16 *kt_at = p.kt + turned, *qt_at = p.qt + turned;
    const float *a_at = p.gates + (bh * p.chunks + end) * 2 * kChunk + tile * 16, *cbeta_at = a_at + kChunk, *carry_at = p.carry + bh * p.chunks + end;
    const int row = tile * 16 + lane4(), steps_left = (int)min<int64_t>(p.steps - p.chunk0 * kChunk, (int64_t)p.chunks * kChunk);
    const T *d_at = at<T>(p.dout, b, (p.chunk0 + end) * kChunk, head) + min(j, p.value_dim - 1);
    Rows d_rows;
    b8 rows[DK / 32][NI], square[2][3], kt[2][NI], qt[2][NI];                  // square: of X^T, or of P turned
    T d[4];
    f4 a, cbeta{};
    float carry;
    const auto load_rows_of = [&]() {
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) load_block(rows[kb], rows_at, kb);
        cbeta = four(cbeta_at, 0);
    };
    // (chunk after chunk, the last one first)
    const auto load_d_of = [&](int n) {
        if (n >= end - 1) d_rows.set(row, p.dout.step, steps_left - n * kChunk);
#pragma unroll
        for (int m = 0; m < 4; ++m) d[m] = d_at[d_rows.apart[m]];
        if (n > 0) d_at -= kChunk * p.dout.step;
        a = four(a_at, 0);
    };
    const auto load_square_of = [&]() {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) load_block(square[kb], square_at, kb);
        if (!FEEDS) a = four(a_at, 0);
    };
    const auto load_turned_of = [&]() {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            load_block(kt[kb], kt_at, kb);
            load_block(qt[kb], qt_at, kb);
        }
        carry = *carry_at;
    };
    // what a chunk's dO gives, into LDS; then the loads of the chunk before it (of chunk `next`, which is the first one again at the end)
    const auto feed = [&](int of) {
        f4 x;
#pragma unroll
        for (int m = 0; m < 4; ++m) x[m] = j < p.value_dim ? (float)d[m] : 0.0f;
        put_block<NI>(sh.o, tile * 16, x);
        put_block(sh.q[of & 1], tile * 16, x * a * p.scale);
    };
    const auto feed_square = [&]() {
        b8 o[2][NI];
        load_block(o[0], sh.o, 0);
        load_block(o[1], sh.o, 1);
        __builtin_amdgcn_sched_barrier(0);
        sh.e[tile][threadIdx.x & 63] = mmp(square[0], o[0], f4{}) + mmp(square[1], o[1], f4{});
    };
    const auto back = [&](bool more) {                   // the pointers of what is a chunk ahead
        if (!more) return;
        square_at -= 3 * Square;
        a_at -= 2 * kChunk;
    };
    if (!FEEDS) __builtin_amdgcn_s_setprio(3);           // the others wait for them
    if (FEEDS) {
        load_d_of((int)end);
        load_square_of();
        back(end > 0);
        feed((int)end);
        load_d_of(max((int)end - 1, 0));
        all_waves();
        feed_square();
        load_square_of();
    } else {
        load_rows_of();
        load_square_of();
        all_waves();
    }
    load_turned_of();
    for (int n = (int)end; n >= 0; --n) {
        const int64_t unit = bh * p.chunks + n;
        if (n > 0) {
            rows_at -= Inputs;
            kt_at -= Inputs;
            qt_at -= Inputs;
            cbeta_at -= 2 * kChunk;
            --carry_at;
        }
        back(FEEDS ? n > 1 : n > 0);
        if (mine) {
            put_block(sh.s, wave * 16, state);
            put(p.ds + unit * DK * p.columns, p.columns, wave * 16, column, state);
        }
        all_waves();
        const auto by_queries = [&] {
            b8 x[2][3];
            load_block(x[0], sh.q[n & 1], 0);
            load_block(x[1], sh.q[n & 1], 1);
            __builtin_amdgcn_sched_barrier(0);
            state = mmp(qt[0], x[0], state * carry) + mmp(qt[1], x[1], f4{});
        };
        if (FEEDS) {
            by_queries();
            feed(n - 1);                                 // (behind the first chunk: once more, for nobody)
            load_d_of(max(n - 2, 0));
        } else {
            const f4 z = sh.e[tile][threadIdx.x & 63];
            put_block(sh.z, tile * 16, z + rows_by(rows, sh.s) * cbeta);
            load_rows_of();
        }
        all_waves();
        if (FEEDS) {
            feed_square();
            load_square_of();
        } else {
            b8 z[2][3];
            load_block(z[0], sh.z, 0);
            load_block(z[1], sh.z, 1);
            __builtin_amdgcn_sched_barrier(0);
            f4 c[4] = {};
            mmp(square[0], z[0], c[0], c[1]);
            mmp(square[1], z[1], c[2], c[3]);
            const f4 y = (c[0] + c[1]) + (c[2] + c[3]);
            put_block(sh.u, tile * 16, -y * a);
            put(p.dy + unit * kChunk * p.columns, p.columns, tile * 16, column, y);
            load_square_of();
        }
        all_waves();
        if (!FEEDS) by_queries();
        b8 u[2][3];
        load_block(u[0], sh.u, 0);
        load_block(u[1], sh.u, 1);
        __builtin_amdgcn_sched_barrier(0);
        state = mmp(kt[0], u[0], state) + mmp(kt[1], u[1], f4{});
        load_turned_of();
    }
    if (mine && not_finite(state)) sh.bad = 1;
    all_waves();
    if (__builtin_amdgcn_readfirstlane(sh.bad)) return false;
    if (mine) put_state(p, bh, wave * 16, j, state);
    return true;
}

template <typename T, int DK>
__device__ void back_chain_by_steps(const DeltaArgs &p, int64_t bh, int slice)
{
    const int64_t b = bh / p.heads, head = bh % p.heads, key = head / p.group;
    Column<DK> c(p, bh, slice);
#pragma unroll 1
    for (int n = p.chunks - 1; n >= 0; --n) {
        const int64_t unit = bh * p.chunks + n, t0 = (p.chunk0 + n) * kChunk;
        c.keep(p.ds + unit * DK * p.columns, p.columns);
#pragma unroll 1
        for (int l = kChunk - 1; l >= 0; --l) {
            const int64_t t = t0 + l, gate = (b * p.steps + t) * p.heads + head;
            float dy = 0.0f;
            if (t < p.steps) {
                const T *const k = at<T>(p.k, b, t, key), *const q = at<T>(p.q, b, t, key);
                const bool cut = p.g[gate] < kNoCarry || (p.reset && p.reset[b * p.steps + t] != 0);
                const float carry = cut ? 0.0f : expf(p.g[gate]), d = c.in ? p.scale * (float)at<T>(p.dout, b, t, head)[c.j] : 0.0f;
                float sk = 0.0f;
#pragma unroll
                for (int i = 0; i < c.R; ++i)
                    if (c.row(i) < p.key_dim) {
                        c.s[i] = fmaf((float)q[c.row(i)], d, c.s[i]);
                        sk = fmaf(c.s[i], (float)k[c.row(i)], sk);
                    }
                sk = column_sum(sk);
                dy = c.in ? p.beta[gate] * sk : 0.0f;
#pragma unroll
                for (int i = 0; i < c.R; ++i)
                    if (c.row(i) < p.key_dim) c.s[i] = cut ? 0.0f : carry * fmaf((float)k[c.row(i)], -dy, c.s[i]);
            }
            if (c.lane == 0) p.dy[(unit * kChunk + l) * p.columns + c.j] = dy;
        }
    }
    c.put_last(p);
}

template <typename T, int DK>
__global__ void __launch_bounds__(512, kPlanes<T> == 1 ? 4 : 2) delta_back_chain_kernel(DeltaArgs p)
{
    __shared__ BackShared<T, DK> sh;
    const int64_t die = blockIdx.x & 7, place = blockIdx.x >> 3, bh = place / p.slices * 8 + die;
    if (bh >= p.batch * p.heads) return;
    const int slice = (int)(place % p.slices);
    const bool finite = threadIdx.x < 256 ? run_back_chain<T, DK, false>(p, sh, bh, slice) : run_back_chain<T, DK, true>(p, sh, bh, slice);
    if (!finite) {
        __syncthreads();                                 // (for what the chain has written, which is written over)
        back_chain_by_steps<T, DK>(arguments_again(), bh, slice);
    }
}

// ---- backward: all gradients at once -------------------------------------------------------------------------------------------
// Over the value dimensions, 64 at a time: dO S^T, dY S^T, Y dS^T (16 key dimensions by a wave) and dO Y^T, dY Y^T; then with the gradient by Q K^T, and after
// it with the one by K K^T, the products over the chunk's steps.  LDS and registers for two workgroups on a compute unit: it waits for memory and barriers
// two thirds of the time (one workgroup: 320 us for 4 x 2048 steps x 16 heads of 128 x 128).  fp16 spills 35 registers so, and is no slower for it: the
// whole pass 864 us, with one workgroup and no spills 874.

__device__ inline float row_sum(float x)
{
    return row_reduce(x, [](float a, float b) { return a + b; });
}

template <int NI>
union BackOutputShared {
    struct {
        __bf16 o[NI * kChunk * kChunk], dy[3 * kChunk * kChunk], y[3 * kChunk * kChunk];
    } in;
    struct {
        __bf16 rows[3 * kChunk * kChunk], turned[3 * kChunk * kChunk];           // the gradient by Q K^T, then the one by K K^T
    } by;
};

// by the first wave, a lane a step: the gradients by the gates, from what their products with everything they decay add up to
__device__ inline void put_gate_gradients(const DeltaArgs &p, const Gates &gates, int64_t b, int64_t head, int64_t t0, double sum, float dbeta)
{
    const int i = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    // the steps from here to the next cut (all behind a cut add up to 0, which their roundings would not)
    for (int step = 1; step < kChunk; step <<= 1) {
        const double later = __shfl_down(sum, step);
        if (i + step < kChunk && gates.part[i + step] == gates.part[i]) sum += later;
    }
    if (t0 + i < p.steps) {
        const int64_t to = (b * p.steps + t0 + i) * p.heads + head;
        p.dg[to] = gates.cut[i] ? 0.0f : (float)sum;
        p.dbeta[to] = dbeta;
    }
}

// a tile on or below the diagonal as the left operand that sums over its columns, and (turned) over its rows
__device__ inline void put_tile(__bf16 *p, __bf16 *turned, int ti, int tj, f4 v)
{
    b4 to[3];
    split(v, to);
    const int i = ti * 16 + lane4(), j = tj * 16 + lane16();
#pragma unroll
    for (int plane = 0; plane < 3; ++plane) {
        *reinterpret_cast<b4 *>(turned + place_in<3>(j, i, 2, plane) + (i & 4)) = to[plane];
#pragma unroll
        for (int m = 0; m < 4; ++m) p[place_in<3>(i + m, j, 2, plane) + (j & 7)] = to[plane][m];
    }
}

// The same again without a product across a cut, for the chunks whose gradients are not all finite: w1 is the gradient by Q K^T, w2 the one by K K^T, w3 the one
// by the decays, all chunk x chunk.  A wave takes a step at a time, a lane its key dimensions.
template <typename T, int DK>
__device__ void gradients_within_cuts(const DeltaArgs &p, Gates &gates, float *w1, float *slope, float *kept, int wave)
{
    const int64_t unit = blockIdx.x;
    float *const w2 = w1 + kChunk * kChunk, *const w3 = w2 + kChunk * kChunk;
    const int64_t bh = unit / p.chunks, chunk = unit % p.chunks, b = bh / p.heads, head = bh % p.heads, key = head / p.group, t0 = (p.chunk0 + chunk) * kChunk;
    const int steps = (int)min<int64_t>(kChunk, p.steps - t0), lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    const int first = gates.part[0] == 0 ? 0 : -1, last = gates.part[kChunk - 1];            // what S0 reaches, and what reaches dS1
    const float *const s = p.s + unit * DK * p.columns, *const ds = p.ds + unit * DK * p.columns;
    const float *const ys = p.y + unit * kChunk * p.columns, *const dys = p.dy + unit * kChunk * p.columns;
    if (wave == 0) gates.sum_within_cuts(p, (b * p.steps + t0 + lane) * p.heads + head, lane, lane < steps);
    __syncthreads();                                     // (and what has been written is written over)
#pragma unroll 1
    for (int u = wave * 64 + lane; u < kChunk * kChunk; u += DK * 4) {
        const int i = u / kChunk, j = u % kChunk;
        float by_qk = 0.0f, by_kk = 0.0f, by_decay = 0.0f;
        if (j <= i && i < steps && gates.part[i] == gates.part[j]) {
            const T *const dout = at<T>(p.dout, b, t0 + i, head), *const q = at<T>(p.q, b, t0 + i, key), *const ki = at<T>(p.k, b, t0 + i, key),
                    *const kj = at<T>(p.k, b, t0 + j, key);
            float from_o = 0.0f, from_y = 0.0f, qk = 0.0f, kk = 0.0f;
#pragma unroll 1
            for (int c = 0; c < p.value_dim; ++c) {
                const float y = ys[j * p.columns + c];
                from_o = fmaf((float)dout[c], y, from_o);
                if (j < i) from_y = fmaf(dys[i * p.columns + c], y, from_y);
            }
#pragma unroll 1
            for (int d = 0; d < p.key_dim; ++d) {
                qk = fmaf((float)q[d], (float)kj[d], qk);
                if (j < i) kk = fmaf((float)ki[d], (float)kj[d], kk);
            }
            const float decay = gates.decay(i, j), o = p.scale * from_o * decay, f = from_y * decay;
            by_qk = o * gates.beta[j];
            by_kk = -f * gates.beta[j];
            by_decay = o * qk - f * kk;
        }
        w1[u] = by_qk;
        w2[u] = by_kk;
        w3[u] = by_decay;
    }
    __syncthreads();
#pragma unroll 1
    for (int i = wave; i < steps; i += DK / 16) {
        const int part = gates.part[i];
        const T *const dout = at<T>(p.dout, b, t0 + i, head), *const qi = at<T>(p.q, b, t0 + i, key), *const ki = at<T>(p.k, b, t0 + i, key);
        float slope_sum = 0.0f, kept_sum = 0.0f;
#pragma unroll 1
        for (int d = lane; d < p.key_dim; d += 64) {
            float o_state = 0.0f, y_state = 0.0f, carried = 0.0f;
#pragma unroll 1
            for (int c = 0; c < p.value_dim; ++c) {
                if (part == first) {
                    o_state = fmaf((float)dout[c], s[d * p.columns + c], o_state);
                    y_state = fmaf(dys[i * p.columns + c], s[d * p.columns + c], y_state);
                }
                if (part == last) carried = fmaf(ys[i * p.columns + c], ds[d * p.columns + c], carried);
            }
            o_state = part == first ? o_state * gates.a[i] * p.scale : 0.0f;
            y_state = part == first ? y_state * gates.a[i] : 0.0f;
            carried = part == last ? carried * gates.c[i] : 0.0f;
            slope_sum += (float)qi[d] * o_state - (float)ki[d] * y_state;
            kept_sum = fmaf((float)ki[d], carried, kept_sum);
            float dq = o_state, dk = (part == last ? carried * gates.beta[i] : 0.0f) - y_state;
#pragma unroll 1
            for (int j = 0; j < steps; ++j) {
                if (gates.part[j] != part) continue;
                const float k = (float)at<T>(p.k, b, t0 + j, key)[d];
                if (j <= i) dq = fmaf(w1[i * kChunk + j], k, dq);
                if (j < i) dk = fmaf(w2[i * kChunk + j], k, dk);
                if (j > i) dk = fmaf(w2[j * kChunk + i], k, dk);
                if (j >= i) dk = fmaf(w1[j * kChunk + i], (float)at<T>(p.q, b, t0 + j, key)[d], dk);
            }
            if (p.group > 1) {
                p.gq[(unit * kChunk + i) * DK + d] = dq;
                p.gk[(unit * kChunk + i) * DK + d] = dk;
            } else {
                out_at<T>(p.dq, b, t0 + i, head)[d] = (T)dq;
                out_at<T>(p.dk, b, t0 + i, head)[d] = (T)dk;
            }
        }
        const auto plus = [](float x, float y) { return x + y; };
        slope_sum = wave_reduce(slope_sum, 0.0f, plus);
        kept_sum = wave_reduce(kept_sum, 0.0f, plus);
        if (lane == 0) slope[i] = slope_sum, kept[i] = kept_sum;
    }
    __syncthreads();
    if (wave != 0) return;
    const int i = lane, part = gates.part[i];
    float dot = 0.0f;                                    // S0 . dS1, where nothing lies between
    if (first == last)
        for (int d = 0; d < p.key_dim; ++d)
            for (int c = lane; c < p.value_dim; c += 64) dot = fmaf(s[d * p.columns + c], ds[d * p.columns + c], dot);
    dot = wave_reduce(dot, 0.0f, [](float x, float y) { return x + y; });
    float dbeta = 0.0f, on = 0.0f;
    double sum = 0.0;
    if (i < steps) {
        float column = 0.0f, row = 0.0f;
        for (int j = 0; j < steps; ++j) {
            if (gates.part[j] != part) continue;
            if (j > i) column += w3[j * kChunk + i];
            if (j < i) row = fmaf(w3[i * kChunk + j], gates.beta[j], row);
        }
        const float beta = gates.beta[i], held = kept[i];
        dbeta = held + column + w3[i * kChunk + i];
        on = part == last ? beta * held : 0.0f;
        sum = (double)(slope[i] + row) - (double)(beta * column) - (double)on;
    }
    double carried_on = on;
    for (int step = 32; step > 0; step >>= 1) carried_on += __shfl_xor(carried_on, step);
    if (i == kChunk - 1) sum += carried_on + (first == last ? (double)gates.a[i] * dot : 0.0);
    put_gate_gradients(p, gates, b, head, t0, sum, dbeta);
}
template <typename T, int DK>
__global__ void __launch_bounds__(DK * 4, DK == 128 ? (kPlanes<T> == 3 ? 2 : 4) : DK == 64 ? 2 : 1) delta_back_output_kernel(DeltaArgs p)
{
    constexpr int NI = kPlanes<T>, W = DK / 16, Most = (kLower + W - 1) / W;
    __shared__ Gates gates;
    __shared__ __attribute__((aligned(16))) BackOutputShared<NI> sh;
    __shared__ float by_row[4][kChunk], by_column[4][kChunk], by_itself[kChunk]; // of the chunk x chunk matrix, by tile; its diagonal, which no decay is in
    __shared__ float by_state[W][kChunk], kept[W][kChunk], dots[W];              // by wave
    __shared__ int32_t again;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = blockIdx.x, bh = unit / p.chunks, chunk = unit % p.chunks, b = bh / p.heads, head = bh % p.heads, key = head / p.group;
    const int64_t t0 = (p.chunk0 + chunk) * kChunk, inputs = ((b * (p.heads / p.group) + key) * p.chunks + chunk) * NI * kChunk * DK;
    gates.load(p, b, head, t0);
    f4 o_state[4] = {}, y_state[4] = {}, carried[4] = {}, from_o[Most] = {}, from_y[Most] = {};
    float dot = 0.0f;
    const float *const s = p.s + unit * DK * p.columns, *const ds = p.ds + unit * DK * p.columns;
    const int row_at = (wave * 16 + lane16()) * p.columns + lane8();
    for (int column = 0; column < p.columns; column += kChunk) {
        __syncthreads();
        for (int u = threadIdx.x; u < kChunk * 8; u += DK * 4) {
            const int row = u / 8, j = u % 8 * 8;
            const bool in = t0 + row < p.steps;
            b8 po[NI], pd[3], py[3];
            planes_of(load_raw(at<T>(p.dout, b, t0 + row, head), in, column + j, p.value_dim), po);
            vec8<float> dy, y;
            const int64_t from = (unit * kChunk + row) * p.columns + column + j;
            __builtin_memcpy(&dy, p.dy + from, 32);
            __builtin_memcpy(&y, p.y + from, 32);
            if (in) {                                    // dv is dy
                T *const to = out_at<T>(p.dv, b, t0 + row, head) + column + j;
                T v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (T)dy[e];
                if (column + j + 8 <= p.value_dim) __builtin_memcpy(to, v, sizeof(v));
                else
                    for (int e = 0; e < 8; ++e)
                        if (column + j + e < p.value_dim) to[e] = v[e];
            }
            split(dy, pd);
            split(y, py);
#pragma unroll
            for (int i = 0; i < NI; ++i) *reinterpret_cast<b8 *>(sh.in.o + place_in<NI>(row, j, 2, i)) = po[i];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                *reinterpret_cast<b8 *>(sh.in.dy + place_in<3>(row, j, 2, i)) = pd[i];
                *reinterpret_cast<b8 *>(sh.in.y + place_in<3>(row, j, 2, i)) = py[i];
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int kb = 0; kb < 2; ++kb) {
            vec8<float> before, after;
            __builtin_memcpy(&before, s + (row_at + column + kb * 32), 32);
            __builtin_memcpy(&after, ds + (row_at + column + kb * 32), 32);
#pragma unroll
            for (int m = 0; m < 8; ++m) dot = fmaf(before[m], after[m], dot);
            b8 right[3], left[3], o[NI];
            split(before, right);
#pragma unroll
            for (int ti = 0; ti < 4; ++ti) {
                load_block(o, sh.in.o, ti * 2 + kb);
                load_block(left, sh.in.dy, ti * 2 + kb);
                o_state[ti] = mmp(o, right, o_state[ti]);
                y_state[ti] = mmp(left, right, y_state[ti]);
            }
            split(after, right);
#pragma unroll
            for (int ti = 0; ti < 4; ++ti) {
                load_block(left, sh.in.y, ti * 2 + kb);
                carried[ti] = mmp(left, right, carried[ti]);
            }
#pragma unroll
            for (int e = 0; e < Most; ++e) {
                const int u = wave + W * e;
                if (u >= kLower) continue;
                int ti, tj;
                lower_tile(u, ti, tj);
                load_block(right, sh.in.y, tj * 2 + kb);
                load_block(o, sh.in.o, ti * 2 + kb);
                load_block(left, sh.in.dy, ti * 2 + kb);
                from_o[e] = mmp(o, right, from_o[e]);
                from_y[e] = mmp(left, right, from_y[e]);
            }
        }
    }
    // q and k of four steps times 16 in this wave's key dimensions (all asked for at once, long before they are used)
    const int col = wave * 16 + lane16();
    b4 qs[4][NI], ks[4][NI];
#pragma unroll
    for (int ti = 0; ti < 4; ++ti) {
        const int64_t from = inputs + place_in<NI>(col, ti * 16 + lane4(), 2, 0) + (lane4() & 4);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            qs[ti][i] = *reinterpret_cast<const b4 *>(p.qt + from + i * 512);
            ks[ti][i] = *reinterpret_cast<const b4 *>(p.kt + from + i * 512);
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < Most; ++e) {
        const int u = wave + W * e;
        if (u >= kLower) continue;
        int ti, tj;
        lower_tile(u, ti, tj);
        f4 qk{}, kk{};
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            b8 left[NI], right[NI];
            load_block(right, p.kp + inputs, tj * (DK / 32) + kb);
            load_block(left, p.qp + inputs, ti * (DK / 32) + kb);
            qk = mmp(left, right, qk);
            load_block(left, p.kp + inputs, ti * (DK / 32) + kb);
            kk = mmp(left, right, kk);
        }
        const int j = tj * 16 + lane16();
        const float beta = gates.beta[j];
        float column_sum = 0.0f;
        f4 by_qk;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int i = ti * 16 + lane4() + m;
            const float decay = gates.decay(i, j);
            const float o = p.scale * from_o[e][m] * decay, f = i > j ? from_y[e][m] * decay : 0.0f, by_decay = o * qk[m] - f * kk[m];
            by_qk[m] = o * beta;
            from_y[e][m] = -f * beta;
            if (i == j) by_itself[i] = by_decay;
            column_sum += i == j ? 0.0f : by_decay;
            const float sum = row_sum(i == j ? 0.0f : by_decay * beta);
            if (lane16() == 0) by_row[tj][i] = sum;
        }
        column_sum += __shfl_xor(column_sum, 16);
        column_sum += __shfl_xor(column_sum, 32);
        if (lane4() == 0) by_column[ti][j] = column_sum;
        put_tile(sh.by.rows, sh.by.turned, ti, tj, by_qk);
        // what a block of 32 has above the diagonal
        if (ti == tj && (ti & 1) == 0) put_tile(sh.by.rows, sh.by.turned, ti, ti + 1, f4{});
    }
#pragma unroll
    for (int ti = 0; ti < 4; ++ti) {
        const f4 a = four(gates.a, ti * 16), c = four(gates.c, ti * 16);
        o_state[ti] *= a * p.scale;
        y_state[ti] *= a;
        carried[ti] *= c;
        f4 q{}, k{};
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            q += __builtin_convertvector(qs[ti][i], f4);
            k += __builtin_convertvector(ks[ti][i], f4);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int i = ti * 16 + lane4() + m;
            const float state_sum = row_sum(q[m] * o_state[ti][m] - k[m] * y_state[ti][m]), kept_sum = row_sum(k[m] * carried[ti][m]);
            if (lane16() == 0) by_state[wave][i] = state_sum, kept[wave][i] = kept_sum;
        }
        carried[ti] = carried[ti] * four(gates.beta, ti * 16) - y_state[ti];
    }
    dot = wave_reduce(dot, 0.0f, [](float x, float z) { return x + z; });
    if ((threadIdx.x & 63) == 0) dots[wave] = dot;
    __syncthreads();
    b8 kt[2][NI], qt[2][NI];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        load_block(kt[kb], p.kt + inputs, wave * 2 + kb);
        load_block(qt[kb], p.qt + inputs, wave * 2 + kb);
    }
#pragma unroll
    for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            b8 x[3];
            if (kb <= ti / 2) {
                load_block(x, sh.by.rows, ti * 2 + kb);
                o_state[ti] = mmp(x, kt[kb], o_state[ti]);
            }
            if (kb >= ti / 2) {
                load_block(x, sh.by.turned, ti * 2 + kb);
                carried[ti] = mmp(x, qt[kb], carried[ti]);
            }
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < Most; ++e) {
        const int u = wave + W * e;
        if (u >= kLower) continue;
        int ti, tj;
        lower_tile(u, ti, tj);
        put_tile(sh.by.rows, sh.by.turned, ti, tj, from_y[e]);
    }
    __syncthreads();
#pragma unroll
    for (int ti = 0; ti < 4; ++ti) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            b8 x[3];
            if (kb <= ti / 2) {
                load_block(x, sh.by.rows, ti * 2 + kb);
                carried[ti] = mmp(x, kt[kb], carried[ti]);
            }
            if (kb >= ti / 2) {
                load_block(x, sh.by.turned, ti * 2 + kb);
                carried[ti] = mmp(x, kt[kb], carried[ti]);
            }
        }
        const f4 dq = o_state[ti], dk = carried[ti];
        if (p.group > 1) {                               // added up over the heads that share the keys by another launch
            put(p.gq + unit * kChunk * DK, DK, ti * 16, wave * 16, dq);
            put(p.gk + unit * kChunk * DK, DK, ti * 16, wave * 16, dk);
        } else if (col < p.key_dim) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int64_t t = t0 + ti * 16 + lane4() + m;
                if (t >= p.steps) continue;
                out_at<T>(p.dq, b, t, head)[col] = (T)dq[m];
                out_at<T>(p.dk, b, t, head)[col] = (T)dk[m];
            }
        }
    }
    if (wave == 0) {
        const int i = threadIdx.x, tile = i >> 4;
        const float beta = gates.beta[i];
        float held = 0.0f, slope = 0.0f, all = 0.0f;
        for (int w = 0; w < W; ++w) held += kept[w][i], slope += by_state[w][i], all += dots[w];
        float column = 0.0f;
        for (int ti = tile; ti < 4; ++ti) column += by_column[ti][i];
        for (int tj = 0; tj <= tile; ++tj) slope += by_row[tj][i];
        const float dbeta = held + column + by_itself[i], on = beta * held;      // on: of what goes on behind the chunk
        double sum = (double)slope - (double)(beta * column) - (double)on, carried_on = on;
        for (int step = 32; step > 0; step >>= 1) carried_on += __shfl_xor(carried_on, step);
        if (i == kChunk - 1) sum += carried_on + (double)gates.a[kChunk - 1] * all;
        // whatever is not finite among the other gradients, or what they are made of, is so in these sums of products with it
        const uint64_t bad = __ballot(!(fabsf((float)sum + dbeta) < INFINITY));
        if (i == 0) again = bad != 0;
        put_gate_gradients(p, gates, b, head, t0, sum, dbeta);
    }
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(again)) gradients_within_cuts<T, DK>(arguments_again(), gates, reinterpret_cast<float *>(&sh), by_state[0], kept[0], wave);
}


// the gradients by queries and keys that heads share: the sum over the heads, in their order
template <typename T>
__global__ void __launch_bounds__(256) delta_group_kernel(DeltaArgs p, int dk)
{
    const int64_t key_heads = p.heads / p.group, unit = blockIdx.x, n = unit % p.chunks, bk = unit / p.chunks, b = bk / key_heads, key = bk % key_heads;
    const int64_t t0 = (p.chunk0 + n) * kChunk;
    for (int u = threadIdx.x; u < kChunk * dk; u += 256) {
        const int row = u / dk, col = u % dk;
        if (t0 + row >= p.steps || col >= p.key_dim) continue;
        float dq = 0.0f, dkey = 0.0f;
        for (int h = 0; h < p.group; ++h) {
            const int64_t from = ((b * p.heads + key * p.group + h) * p.chunks + n) * kChunk * dk + u;
            dq += p.gq[from];
            dkey += p.gk[from];
        }
        out_at<T>(p.dq, b, t0 + row, key)[col] = (T)dq;
        out_at<T>(p.dk, b, t0 + row, key)[col] = (T)dkey;
    }
}

// ---- a few steps, one by one --------------------------------------------------------------------------------------------------
// A workgroup has 64 columns of a head's state in registers: 16 groups of lanes, every 16th row each, a lane four columns.  S^T k and S^T q are
// summed together, so a step has one barrier: o = e^g S^T q + (k . q) beta y.

template <typename T, int DK>
__global__ void __launch_bounds__(256) delta_step_kernel(DeltaArgs p)
{
    constexpr int R = DK / 16;
    __shared__ f4 sums[2][2][4][16];                     // [step parity][S^T k, S^T q][wave][columns]
    __shared__ float kq_part[2][4];
    const int tiles = p.columns / 64, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = threadIdx.x >> 4;
    const int64_t bh = blockIdx.x / tiles, b = bh / p.heads, head = bh % p.heads;
    const int j = blockIdx.x % tiles * 64 + (lane & 15) * 4;
    const bool whole = j + 4 <= p.value_dim;
    f4 s[R];
    const int64_t base = bh * p.key_dim * p.value_dim + j;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = group + 16 * i;
        s[i] = f4{};
        if (!p.state || row >= p.key_dim) continue;
        const float *const from = p.state + base + (int64_t)row * p.value_dim;
        if (whole) __builtin_memcpy(&s[i], from, 16);
        else
            for (int m = 0; m < 4; ++m)
                if (j + m < p.value_dim) s[i][m] = from[m];
    }
    for (int64_t t = 0; t < p.steps; ++t) {
        const T *const kt = at<T>(p.k, b, t, head / p.group), *const qt = at<T>(p.q, b, t, head / p.group), *const vt = at<T>(p.v, b, t, head) + j;
        const int64_t gate = (b * p.steps + t) * p.heads + head;
        const float g = p.g[gate], beta = p.beta[gate];
        const bool cut = g < kNoCarry || (p.reset && p.reset[b * p.steps + t] != 0);
        const float carry = cut ? 0.0f : expf(g);
        float k[R], q[R];
        f4 v{};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = group + 16 * i;
            k[i] = row < p.key_dim ? (float)kt[row] : 0.0f;
            q[i] = row < p.key_dim ? (float)qt[row] : 0.0f;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
            if (j + m < p.value_dim) v[m] = (float)vt[m];
        if (cut)
#pragma unroll
            for (int i = 0; i < R; ++i) s[i] = f4{};
        f4 sk{}, sq{};
        float kq = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int m = 0; m < 4; ++m) sk[m] = fmaf(s[i][m], k[i], sk[m]), sq[m] = fmaf(s[i][m], q[i], sq[m]);
            kq = fmaf(k[i], q[i], kq);
        }
        for (int d = 16; d < 64; d <<= 1) {
#pragma unroll
            for (int m = 0; m < 4; ++m) sk[m] += __shfl_xor(sk[m], d), sq[m] += __shfl_xor(sq[m], d);
            kq += __shfl_xor(kq, d);
        }
        const int turn = t & 1;
        if (lane < 16) sums[turn][0][wave][lane] = sk, sums[turn][1][wave][lane] = sq;
        if (lane == 0) kq_part[turn][wave] = kq;
        __syncthreads();
        sk = sq = f4{};
        kq = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) sk += sums[turn][0][w][lane & 15], sq += sums[turn][1][w][lane & 15], kq += kq_part[turn][w];
        const f4 u = beta * (v - carry * sk);
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = s[i] * carry + k[i] * u;
        if (threadIdx.x < 16) {
            const f4 o = p.scale * (carry * sq + kq * u);
            T *const to = out_at<T>(p.o, b, t, head) + j;
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if (j + m < p.value_dim) to[m] = (T)o[m];
        }
    }
    if (!p.last) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = group + 16 * i;
        if (row >= p.key_dim) continue;
        float *const to = p.last + base + (int64_t)row * p.value_dim;
        if (whole) __builtin_memcpy(to, &s[i], 16);
        else
            for (int m = 0; m < 4; ++m)
                if (j + m < p.value_dim) to[m] = s[i][m];
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

// Up to so many steps are taken one by one.  (One by one and in chunks, us: 32 heads of 128 x 128 in bf16 6 steps 19.0 and 18.1, 8 23.9 and 18.0; 16 of 64 x 64 6
// 13.4 and 15.1, 8 17.0 and 15.1; one of 16 x 16 8 12.3 and 13.3, 10 14.9 and 13.2.  256 of 128 x 128 12 37.7 and 40.1, 16 48.3 and 39.5; 2048 12 254 and 280, 16 326
// and 279; 4096 of 32 x 32 16 138 and 146, 24 207 and 155.)
int64_t few_steps(int64_t batch, int64_t heads) { return batch * heads >= 256 ? 16 : 6; }
// Workspace of the chunks that a launch takes, counted as for fp32 and keys that are not shared: bf16 touches half of it, with two heads a key three eighths.
// Forward: 8191 steps x 32 heads in 96, 192, 384, 768 MB, us: bf16 418, 391, 386, 399 (two heads a key 399, 361, 348, 374); fp16 619, 589, 666, 656; fp32 702, 737, 805, 781.
// Backward: more, as the states before every segment but the first cost a forward pass without outputs (4 x 2048 steps x 16 heads in 256 MB, 512 MB, 1 GB, 2 GB: bf16
// 742, 717, 615, 617; fp32 1214, 1255, 1040, 1041).  A chunk of every head is held at least, however many heads there are.
constexpr int64_t kSegmentBytes = 384ll << 20, kBackSegmentBytes = 2ll << 30;
thread_local int64_t g_segment_bytes = -1;

int padded_key(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }

struct DeltaPlan {
    int64_t chunks, segment, segments, units;            // chunks of a sequence, of a segment; units: (head, chunk) of a segment
    int dk, columns;
    int64_t y, s, dy, ds, gq, gk, carry, gates, spare, xp, pp, xt, kp, qp, kt, qt, bounds, way, total;       // places in the workspace; way: the gradient by the state between segments
};
DeltaPlan plan_delta(const rls_delta_shape &h, bool backward)
{
    DeltaPlan P{};
    P.dk = padded_key(h.key_dim);
    P.columns = (int)align_up(h.value_dim, 64);
    P.chunks = (h.steps + kChunk - 1) / kChunk;
    if (P.chunks == 0 || (!backward && h.steps <= few_steps(h.batch, h.heads))) return P;
    const int64_t bh = h.batch * h.heads, side = kChunk * (int64_t)P.dk, rows = kChunk * (int64_t)P.columns, state = (int64_t)P.dk * P.columns;
    const bool shared = h.heads != h.key_heads;
    const int64_t planes = 3, square = kChunk * kChunk;          // (as for fp32: the workspace does not go by the type)
    const int64_t each = 2 * (6 * square + 3 * planes * side) + (backward ? 2 * (3 * square + planes * side) + 4 * (2 * rows + 2 * state + (shared ? 2 * side : 0)) : 0);
    const int64_t limit = g_segment_bytes >= 0 ? g_segment_bytes : backward ? kBackSegmentBytes : kSegmentBytes, most = std::max<int64_t>(1, limit / each / bh);
    P.segments = (P.chunks + most - 1) / most;
    P.segment = (P.chunks + P.segments - 1) / P.segments;
    P.segments = (P.chunks + P.segment - 1) / P.segment;
    P.units = bh * P.segment;
    int64_t at = 0;
    const auto take = [&](int64_t floats) { const int64_t here = at; at += align_up(floats * 4, 256); return here; };
    P.carry = take(P.units);
    P.gates = take(P.units * 2 * kChunk);
    P.spare = take(64);
    P.xp = take(P.units * 3 * square / 2);
    P.pp = take(P.units * 3 * square / 2);
    const int64_t inputs = P.units / (h.heads / h.key_heads) * planes * side / 2;
    P.kp = take(inputs);
    P.qp = take(inputs);
    P.kt = take(inputs);
    if (backward) {
        P.xt = take(P.units * 3 * square / 2);
        P.qt = take(inputs);
        P.y = take(P.units * rows);
        P.s = take(P.units * state);
        P.dy = take(P.units * rows);
        P.ds = take(P.units * state);
        if (shared) P.gq = take(P.units * side), P.gk = take(P.units * side);
        if (P.segments > 1) {
            P.bounds = take((P.segments - 1) * bh * h.key_dim * h.value_dim);
            P.way = take(2 * bh * h.key_dim * h.value_dim);
        }
    } else if (P.segments > 1) {
        P.way = take(2 * bh * h.key_dim * h.value_dim);
    }
    P.total = at;
    return P;
}

void set_workspace(DeltaArgs &p, const DeltaPlan &P, char *ws)
{
    const auto to = [&](int64_t place) { return reinterpret_cast<float *>(ws + place); };
    p.y = to(P.y); p.s = to(P.s); p.dy = to(P.dy); p.ds = to(P.ds); p.gq = to(P.gq); p.gk = to(P.gk);
    p.carry = to(P.carry); p.gates = to(P.gates); p.spare = to(P.spare);
    const auto planes = [&](int64_t place) { return reinterpret_cast<__bf16 *>(ws + place); };
    p.xp = planes(P.xp); p.pp = planes(P.pp); p.xt = planes(P.xt);
    p.kp = planes(P.kp); p.qp = planes(P.qp); p.kt = planes(P.kt); p.qt = planes(P.qt);
    p.columns = P.columns;
}

template <typename T, int DK>
struct DeltaLaunch {
    static void prepare(const DeltaArgs &p, hipStream_t s)
    {
        hipLaunchKernelGGL((delta_prepare_kernel<T, DK>), dim3((unsigned)(p.batch * p.heads * p.chunks)), dim3(256), 0, s, p);
    }
    static unsigned slices(const DeltaArgs &p) { return (unsigned)((p.batch * p.heads + 7) / 8 * 8 * p.slices); }
    static void chain(const DeltaArgs &p, bool keep, hipStream_t s)
    {
        auto *const kernel = keep ? delta_chain_kernel<T, DK, true> : delta_chain_kernel<T, DK, false>;
        hipLaunchKernelGGL(kernel, dim3(slices(p)), dim3(512), 0, s, p);
    }
    static hipError_t forward(DeltaArgs p, const DeltaPlan &P, float *way, hipStream_t s)
    {
        if (p.steps <= few_steps(p.batch, p.heads)) {
            p.columns = P.columns;
            hipLaunchKernelGGL((delta_step_kernel<T, DK>), dim3((unsigned)(p.batch * p.heads * (p.columns / 64))), dim3(256), 0, s, p);
            return hipGetLastError();
        }
        const int64_t state = p.batch * p.heads * p.key_dim * p.value_dim;
        float *const last = p.last;
        p.slices = (p.value_dim + 15) / 16;
        for (int64_t seg = 0; seg < P.segments; ++seg) {
            p.chunk0 = seg * P.segment;
            p.chunks = (int32_t)std::min(P.segment, P.chunks - p.chunk0);
            p.last = seg + 1 < P.segments ? way + (seg & 1) * state : last;
            prepare(p, s);
            chain(p, false, s);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            p.state = p.last;
        }
        return hipSuccess;
    }
    // The states before the segments first (nothing to do with one segment), then the segments from the last to the first
    static hipError_t backward(DeltaArgs p, const DeltaPlan &P, const float *dlast, float *dstate, float *bounds, float *way, hipStream_t s)
    {
        const int64_t state = p.batch * p.heads * p.key_dim * p.value_dim;
        const float *const first = p.state;
        p.keep = 1;
        p.slices = p.columns / 16;                       // (what is kept is read up to the last of the columns)
        for (int64_t seg = 0; seg + 1 < P.segments; ++seg) {
            p.chunk0 = seg * P.segment;
            p.chunks = (int32_t)P.segment;
            p.state = seg == 0 ? first : bounds + (seg - 1) * state;
            p.last = bounds + seg * state;
            prepare(p, s);
            chain(p, true, s);
        }
        for (int64_t seg = P.segments - 1; seg >= 0; --seg) {
            p.chunk0 = seg * P.segment;
            p.chunks = (int32_t)std::min(P.segment, P.chunks - p.chunk0);
            p.state = seg == 0 ? first : bounds + (seg - 1) * state;
            p.last = nullptr;
            prepare(p, s);
            chain(p, true, s);
            const dim3 grid((unsigned)(p.batch * p.heads * p.chunks));
            DeltaArgs back = p;
            back.state = dlast;
            back.last = seg > 0 ? way + (seg & 1) * state : dstate;
            hipLaunchKernelGGL((delta_back_chain_kernel<T, DK>), dim3(slices(p)), dim3(512), 0, s, back);
            dlast = back.last;
            hipLaunchKernelGGL((delta_back_output_kernel<T, DK>), grid, dim3(DK * 4), 0, s, p);
            if (p.group > 1)
                hipLaunchKernelGGL(delta_group_kernel<T>, dim3((unsigned)(p.batch * (p.heads / p.group) * p.chunks)), dim3(256), 0, s, p, DK);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
};

template <typename T, typename F>
hipError_t by_key_dim(int dk, F f)
{
    return dk == 32 ? f(DeltaLaunch<T, 32>{}) : dk == 64 ? f(DeltaLaunch<T, 64>{}) : f(DeltaLaunch<T, 128>{});
}
template <typename F>
hipError_t by_shape(const rls_delta_shape &h, const DeltaPlan &P, F f)
{
    return h.type == RLS_F32 ? by_key_dim<float>(P.dk, f) : h.type == RLS_BF16 ? by_key_dim<__bf16>(P.dk, f) : by_key_dim<_Float16>(P.dk, f);
}

int32_t check_delta(const rls_delta_shape *h)
{
    if (!h) return RLS_ERR_NULL;
    if (h->batch < 1 || h->steps < 0 || h->heads < 1 || h->key_heads < 1 || h->key_dim < 1 || h->value_dim < 1 || !is_type(h->type)) return RLS_ERR_INVALID_ARG;
    if (h->key_dim > RLS_MAX_KEY_DIM || h->value_dim > RLS_MAX_VALUE_DIM || h->steps > RLS_MAX_N || h->batch > (1 << 17) ||
        h->batch * h->heads > (1 << 17) || h->batch * h->steps > (1 << 30))
        return RLS_ERR_INVALID_ARG;
    return h->heads % h->key_heads != 0 ? RLS_ERR_SHAPE : RLS_OK;
}

// an array of heads: bytes from its first to its last element, and whether it stays clear of itself
struct Reach {
    uintptr_t from = 0, to = 0;
    bool meets(const Reach &o) const { return from < o.to && o.from < to; }
};
Reach reach(const void *p, int64_t bytes) { return {(uintptr_t)p, p ? (uintptr_t)p + (uintptr_t)bytes : (uintptr_t)p}; }
int32_t check_heads(const rls_delta_shape &h, const rls_heads *x, int32_t heads, int32_t dim, bool written, Reach *r)
{
    if (!x) return RLS_ERR_NULL;
    if (h.steps > 0 && !x->data_dev) return RLS_ERR_NULL;
    if (x->batch_stride < 0 || x->step_stride < 0 || x->head_stride < 0) return RLS_ERR_SHAPE;
    if (h.steps == 0) return RLS_OK;
    struct { int64_t apart, count; } d[3] = {{x->batch_stride, h.batch}, {x->step_stride, h.steps}, {x->head_stride, heads}};
    int64_t last = dim;
    for (const auto &e : d) {
        if (e.count == 1) continue;
        if (e.apart > (1ll << 40) / (e.count - 1)) return RLS_ERR_SHAPE;        // (no memory reaches that far)
        last += (e.count - 1) * e.apart;
    }
    *r = reach(x->data_dev, last * type_bytes(h.type));
    if (!written) return RLS_OK;
    std::sort(d, d + 3, [](const auto &p, const auto &q) { return p.apart < q.apart; });
    int64_t width = dim;
    for (const auto &e : d) {
        if (e.count == 1) continue;
        if (e.apart < width) return RLS_ERR_SHAPE;
        width = e.apart * (e.count - 1) + width;
    }
    return RLS_OK;
}
Heads heads_of(const rls_heads *x) { return {x->data_dev, x->batch_stride, x->step_stride, x->head_stride}; }

int32_t apart(std::initializer_list<Reach> written, std::initializer_list<Reach> read)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (const Reach &r : read)
            if (w->meets(r)) return RLS_ERR_SHAPE;
        for (auto v = written.begin(); v != w; ++v)
            if (w->meets(*v)) return RLS_ERR_SHAPE;
    }
    return RLS_OK;
}

DeltaArgs args_of(const rls_delta_shape &h, const rls_heads *q, const rls_heads *k, const rls_heads *v, const float *g, const float *beta, const uint8_t *reset)
{
    DeltaArgs p{};
    p.q = heads_of(q); p.k = heads_of(k); p.v = heads_of(v);
    p.g = g; p.beta = beta; p.reset = reset;
    p.batch = h.batch; p.steps = h.steps; p.heads = h.heads; p.group = h.heads / h.key_heads;
    p.key_dim = h.key_dim; p.value_dim = h.value_dim; p.scale = h.scale;
    return p;
}

int32_t check_workspace(int64_t need, const void *ws, int64_t bytes)
{
    return need > 0 && (!ws || (uintptr_t)ws % 256 != 0 || bytes < need) ? RLS_ERR_WORKSPACE : RLS_OK;
}

__global__ void __launch_bounds__(256) delta_copy_kernel(const float *from, float *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from ? from[i] : 0.0f;
}
hipError_t copy_state(const float *from, float *to, int64_t n, hipStream_t s)
{
    if (to && to != from) hipLaunchKernelGGL(delta_copy_kernel, dim3((unsigned)std::min<int64_t>(4096, (n + 255) / 256)), dim3(256), 0, s, from, to, n);
    return hipGetLastError();
}

}  // namespace

}  // namespace rls

using namespace rls;

extern "C" {

int32_t rls_delta_segment_bytes(int64_t bytes)
{
    g_segment_bytes = bytes < 0 ? -1 : bytes;
    return RLS_OK;
}

int64_t rls_delta_segment_chunks(const rls_delta_shape *shape, int32_t backward)
{
    const int32_t rc = check_delta(shape);
    return rc != RLS_OK ? rc : plan_delta(*shape, backward != 0).segment;
}

int64_t rls_gated_delta_workspace_bytes(const rls_delta_shape *shape, int32_t backward)
{
    const int32_t rc = check_delta(shape);
    return rc != RLS_OK ? rc : plan_delta(*shape, backward != 0).total;
}

int32_t rls_gated_delta(const rls_delta_shape *shape, const rls_heads *q, const rls_heads *k, const rls_heads *v, const float *g_dev, const float *beta_dev,
                        const float *state_dev, const uint8_t *reset_dev, const rls_heads *o, float *last_dev, void *workspace_dev, int64_t workspace_bytes,
                        void *stream)
{
    int32_t rc = check_delta(shape);
    if (rc != RLS_OK) return rc;
    const rls_delta_shape &h = *shape;
    if (h.steps > 0 && (!g_dev || !beta_dev)) return RLS_ERR_NULL;
    Reach rq, rk, rv, ro;
    rc = check_heads(h, q, h.key_heads, h.key_dim, false, &rq);
    if (rc == RLS_OK) rc = check_heads(h, k, h.key_heads, h.key_dim, false, &rk);
    if (rc == RLS_OK) rc = check_heads(h, v, h.heads, h.value_dim, false, &rv);
    if (rc == RLS_OK) rc = check_heads(h, o, h.heads, h.value_dim, true, &ro);
    if (rc != RLS_OK) return rc;
    const DeltaPlan P = plan_delta(h, false);
    rc = check_workspace(P.total, workspace_dev, workspace_bytes);
    if (rc != RLS_OK) return rc;
    const int64_t gates = h.batch * h.steps * h.heads * 4, state = h.batch * h.heads * (int64_t)h.key_dim * h.value_dim;
    const Reach rs = reach(state_dev, state * 4), rl = reach(last_dev, state * 4), rw = reach(workspace_dev, P.total);
    rc = apart({ro, rl, rw}, {rq, rk, rv, reach(g_dev, gates), reach(beta_dev, gates), reach(reset_dev, h.batch * h.steps)});
    if (rc == RLS_OK) rc = apart({ro, last_dev == state_dev ? Reach{} : rl, rw}, {rs});
    if (rc != RLS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    if (h.steps == 0) {
        RLS_HIP_TRY(copy_state(state_dev, last_dev, state, s));
        return RLS_OK;
    }
    DeltaArgs p = args_of(h, q, k, v, g_dev, beta_dev, reset_dev);
    p.o = heads_of(o);
    p.state = state_dev;
    p.last = last_dev;
    set_workspace(p, P, static_cast<char *>(workspace_dev));
    float *const way = reinterpret_cast<float *>(static_cast<char *>(workspace_dev) + P.way);
    RLS_HIP_TRY(by_shape(h, P, [&](auto launch) { return launch.forward(p, P, way, s); }));
    return RLS_OK;
}

int32_t rls_gated_delta_backward(const rls_delta_shape *shape, const rls_heads *q, const rls_heads *k, const rls_heads *v, const float *g_dev,
                                 const float *beta_dev, const float *state_dev, const uint8_t *reset_dev, const rls_heads *dout, const float *dlast_dev,
                                 const rls_heads *dq, const rls_heads *dk, const rls_heads *dv, float *dg_dev, float *dbeta_dev, float *dstate_dev,
                                 void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int32_t rc = check_delta(shape);
    if (rc != RLS_OK) return rc;
    const rls_delta_shape &h = *shape;
    if (h.steps > 0 && (!g_dev || !beta_dev || !dg_dev || !dbeta_dev)) return RLS_ERR_NULL;
    Reach rq, rk, rv, ro, tq, tk, tv;
    rc = check_heads(h, q, h.key_heads, h.key_dim, false, &rq);
    if (rc == RLS_OK) rc = check_heads(h, k, h.key_heads, h.key_dim, false, &rk);
    if (rc == RLS_OK) rc = check_heads(h, v, h.heads, h.value_dim, false, &rv);
    if (rc == RLS_OK) rc = check_heads(h, dout, h.heads, h.value_dim, false, &ro);
    if (rc == RLS_OK) rc = check_heads(h, dq, h.key_heads, h.key_dim, true, &tq);
    if (rc == RLS_OK) rc = check_heads(h, dk, h.key_heads, h.key_dim, true, &tk);
    if (rc == RLS_OK) rc = check_heads(h, dv, h.heads, h.value_dim, true, &tv);
    if (rc != RLS_OK) return rc;
    const DeltaPlan P = plan_delta(h, true);
    rc = check_workspace(P.total, workspace_dev, workspace_bytes);
    if (rc != RLS_OK) return rc;
    const int64_t gates = h.batch * h.steps * h.heads * 4, state = h.batch * h.heads * (int64_t)h.key_dim * h.value_dim;
    const Reach rl = reach(dlast_dev, state * 4), ts = reach(dstate_dev, state * 4), tg = reach(dg_dev, gates), tb = reach(dbeta_dev, gates),
                rw = reach(workspace_dev, P.total);
    rc = apart({tq, tk, tv, tg, tb, ts, rw},
               {rq, rk, rv, ro, reach(g_dev, gates), reach(beta_dev, gates), reach(reset_dev, h.batch * h.steps), reach(state_dev, state * 4)});
    if (rc == RLS_OK) rc = apart({tq, tk, tv, tg, tb, dstate_dev == dlast_dev ? Reach{} : ts, rw}, {rl});
    if (rc != RLS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    if (h.steps == 0) {
        RLS_HIP_TRY(copy_state(dlast_dev, dstate_dev, state, s));
        return RLS_OK;
    }
    DeltaArgs p = args_of(h, q, k, v, g_dev, beta_dev, reset_dev);
    p.dout = heads_of(dout); p.dq = heads_of(dq); p.dk = heads_of(dk); p.dv = heads_of(dv);
    p.dg = dg_dev; p.dbeta = dbeta_dev; p.state = state_dev;
    char *const ws = static_cast<char *>(workspace_dev);
    set_workspace(p, P, ws);
    float *const bounds = reinterpret_cast<float *>(ws + P.bounds), *const way = reinterpret_cast<float *>(ws + P.way);
    RLS_HIP_TRY(by_shape(h, P, [&](auto launch) { return launch.backward(p, P, dlast_dev, dstate_dev, bounds, way, s); }));
    return RLS_OK;
}

}  // extern "C"
