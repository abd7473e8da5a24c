// adamw.cu -- resbm_adamw_step and resbm_grad_norm: one pass over many tensors a launch (include/resbm_train.h).
//
// Both are bound by memory: a step with 32-bit states moves 22 bytes an element (bf16 weight and gradient), one
// with 8-bit states 10. The list of tensors travels as the launch's parameter (up to 448 tensors, 31 KB), so that
// nothing is copied to the device and a captured launch carries its own list.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "abi.h"
#include "common.cuh"
#include "fp8.cuh"
#include "resbm_train.h"

namespace resbm {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlock = RESBM_STATE_BLOCK;             // elements a warp takes at a time: one block of 8-bit states
constexpr int kSmall = 32, kLarge = 448;              // tensors a launch, by the parameter's size
constexpr int kNormGrid = 1216;                       // most CTAs of the gradients' norm: eight on each of 152 SMs
constexpr uint64_t kMagic = 0x7265736264616d77ull;

// The tensors of one launch. A unit is what one CTA takes: kWarps * passes blocks of one tensor.
template <int CAP> struct Table {
    void *w[CAP];
    const void *g[CAP];
    void *m[CAP], *v[CAP];
    float *ms[CAP], *vs[CAP];
    float *master[CAP];
    int64_t n[CAP];
    uint32_t first[CAP + 1];      // a tensor's first unit; first[count]: all units
    uint32_t vec[(CAP + 31) / 32];   // whether everything of a tensor is aligned to four elements
    int32_t count, passes;
};
static_assert(sizeof(Table<kLarge>) <= 32000, "the launch's parameters are at most 32764 bytes");

struct Plan {
    uint64_t magic;
    int64_t tables;               // Table<kSmall> if small, else Table<kLarge>, one after the other behind this
    int32_t small, w_dtype, g_dtype, state, master, pad;
};
static_assert(sizeof(Plan) % 8 == 0, "tables start aligned");

struct Step {
    float b1, omb1, b2, omb2;     // beta and 1 - beta
    float step_size;              // lr / (1 - beta1^t)
    float root;                   // 1 / sqrt(1 - beta2^t)
    float eps, decay;             // decay: 1 - lr weight_decay
    float lr, wd, lnb1, lnb2, t;  // for the values that the device gives
    const float *lr_dev;
    const int64_t *step_dev;
    const float *grad_scale;
};

// Eight elements of a warp's block: with VEC lane l has 4 l .. 4 l + 3 of either half (whole sectors for every
// element size), else l, l + 32, ... below `rem`.
template <bool VEC> __device__ __forceinline__ int elem(int lane, int j)
{
    return VEC ? (j >> 2) * 128 + lane * 4 + (j & 3) : j * 32 + lane;
}
template <bool VEC> __device__ __forceinline__ void load8(const float *p, int lane, int rem, float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float4 u = *reinterpret_cast<const float4 *>(p + k * 128 + lane * 4);
            x[4 * k] = u.x; x[4 * k + 1] = u.y; x[4 * k + 2] = u.z; x[4 * k + 3] = u.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j * 32 + lane < rem ? p[j * 32 + lane] : 0.0f;
    }
}
template <bool VEC> __device__ __forceinline__ void load8(const __nv_bfloat16 *p, int lane, int rem, float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint2 u = *reinterpret_cast<const uint2 *>(p + k * 128 + lane * 4);
            x[4 * k] = __uint_as_float(u.x << 16);
            x[4 * k + 1] = __uint_as_float(u.x & 0xFFFF0000u);
            x[4 * k + 2] = __uint_as_float(u.y << 16);
            x[4 * k + 3] = __uint_as_float(u.y & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j * 32 + lane < rem ? to_f32(p[j * 32 + lane]) : 0.0f;
    }
}
template <bool VEC> __device__ __forceinline__ void load8(const uint8_t *p, int lane, int rem, float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float4 u = from_e4m3x4(*reinterpret_cast<const uint32_t *>(p + k * 128 + lane * 4));
            x[4 * k] = u.x; x[4 * k + 1] = u.y; x[4 * k + 2] = u.z; x[4 * k + 3] = u.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j * 32 + lane < rem ? from_e4m3(p[j * 32 + lane]) : 0.0f;
    }
}
template <bool VEC> __device__ __forceinline__ void store8(float *p, int lane, int rem, const float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            *reinterpret_cast<float4 *>(p + k * 128 + lane * 4) = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < rem) p[j * 32 + lane] = x[j];
    }
}
template <bool VEC> __device__ __forceinline__ void store8(__nv_bfloat16 *p, int lane, int rem, const float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(x[4 * k], x[4 * k + 1]), b = __floats2bfloat162_rn(x[4 * k + 2], x[4 * k + 3]);
            *reinterpret_cast<uint2 *>(p + k * 128 + lane * 4) =
                make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < rem) p[j * 32 + lane] = from_f32<__nv_bfloat16>(x[j]);
    }
}
// (values in units of their scale)
template <bool VEC> __device__ __forceinline__ void store8(uint8_t *p, int lane, int rem, const float (&x)[8])
{
    if (VEC) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            *reinterpret_cast<uint32_t *>(p + k * 128 + lane * 4) = e4m3x4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < rem) p[j * 32 + lane] = e4m3x1(x[j]);
    }
}

// One block of 256 elements (or the last `rem` of a tensor) by one warp. The products of the running means are
// rounded one by one: a fused multiply-add would move values next to a rounding border of e4m3 across it, and
// the same step would then depend on the compiler's contractions.
template <typename W, typename G, bool MASTER, int BITS, bool VEC>
__device__ __forceinline__ void adamw_block(W *w, const G *g, void *mp, void *vp, float *ms, float *vs, float *master,
                                            int lane, int rem, const Step &h, float c)
{
    using S = typename std::conditional<BITS == 8, uint8_t, float>::type;
    S *const m8 = static_cast<S *>(mp), *const v8 = static_cast<S *>(vp);
    float x[8], dg[8], m[8], v[8];
    if (MASTER) load8<VEC>(static_cast<const float *>(master), lane, rem, x);
    else load8<VEC>(static_cast<const W *>(w), lane, rem, x);
    load8<VEC>(g, lane, rem, dg);
    load8<VEC>(static_cast<const S *>(m8), lane, rem, m);
    load8<VEC>(static_cast<const S *>(v8), lane, rem, v);
    float sm = 1.0f, sv = 1.0f;
    if (BITS == 8) {
        sm = *ms;
        sv = *vs;
    }
    uint32_t am = 0, av = 0;   // the largest |m| and sqrt(v), as bits
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float gj = __fmul_rn(dg[j], c);
        if (BITS == 8) {
            m[j] = __fmul_rn(m[j], sm);
            v[j] = __fmul_rn(v[j], sv);
            v[j] = __fmul_rn(v[j], v[j]);
        }
        m[j] = __fadd_rn(__fmul_rn(m[j], h.b1), __fmul_rn(gj, h.omb1));
        v[j] = __fadd_rn(__fmul_rn(v[j], h.b2), __fmul_rn(__fmul_rn(gj, gj), h.omb2));
        const float r = __fsqrt_rn(v[j]);
        x[j] = fmaf(-h.step_size, m[j] / fmaf(r, h.root, h.eps), x[j] * h.decay);
        if (BITS == 8) {
            v[j] = r;
            am = max(am, abs_bits(m[j]));
            av = max(av, abs_bits(r));
        }
    }
    if (MASTER) store8<VEC>(master, lane, rem, x);
    store8<VEC>(w, lane, rem, x);
    if (BITS == 8) {
        const E4m3Scale a = e4m3_scale(__reduce_max_sync(0xffffffffu, am)), b = e4m3_scale(__reduce_max_sync(0xffffffffu, av));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = __fmul_rn(m[j], a.inv);
            // a sqrt(v) above zero keeps a code above zero (and a NaN stays one)
            const float r = __fmul_rn(v[j], b.inv);
            v[j] = v[j] > 0.0f && r < kE4m3Least ? kE4m3Least : r;
        }
        if (lane == 0) {
            *ms = a.scale;
            *vs = b.scale;
        }
    }
    store8<VEC>(m8, lane, rem, m);
    store8<VEC>(v8, lane, rem, v);
}

// The tensor that unit `u` belongs to
template <int CAP> __device__ __forceinline__ int tensor_of(const Table<CAP> &tab, uint32_t u)
{
    int lo = 0, hi = tab.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab.first[mid] <= u) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename W, typename G, bool MASTER, int BITS, int CAP>
__global__ void __launch_bounds__(kThreads) k_adamw(const __grid_constant__ Table<CAP> tab, const __grid_constant__ Step given)
{
    Step h = given;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = tensor_of(tab, blockIdx.x);
    const int64_t n = tab.n[i];
    int64_t b = (int64_t)(blockIdx.x - tab.first[i]) * tab.passes * kWarps + warp;
    const bool vec = (tab.vec[i >> 5] >> (i & 31)) & 1u;
    griddep_wait();
    griddep_launch_dependents();
    float c = 1.0f;
    if (h.grad_scale) {
        c = *h.grad_scale;
        if (!isfinite(c)) return;
    }
    if (h.lr_dev || h.step_dev) {
        const float lr = h.lr_dev ? *h.lr_dev : h.lr;
        const float t = h.step_dev ? (float)*h.step_dev : h.t;
        h.step_size = lr / -expm1f(t * h.lnb1);
        h.root = 1.0f / sqrtf(-expm1f(t * h.lnb2));
        h.decay = 1.0f - lr * h.wd;
    }
    for (int p = 0; p < tab.passes; ++p, b += kWarps) {
        const int64_t at = b * kBlock;
        if (at >= n) return;
        const int rem = n - at < kBlock ? (int)(n - at) : kBlock;
        W *const w = static_cast<W *>(tab.w[i]) + at;
        const G *const g = static_cast<const G *>(tab.g[i]) + at;
        char *const m = static_cast<char *>(tab.m[i]) + at * (BITS / 8), *const v = static_cast<char *>(tab.v[i]) + at * (BITS / 8);
        float *const ms = BITS == 8 ? tab.ms[i] + b : nullptr, *const vs = BITS == 8 ? tab.vs[i] + b : nullptr;
        float *const master = MASTER ? tab.master[i] + at : nullptr;
        if (vec && rem == kBlock) adamw_block<W, G, MASTER, BITS, true>(w, g, m, v, ms, vs, master, lane, rem, h, c);
        else adamw_block<W, G, MASTER, BITS, false>(w, g, m, v, ms, vs, master, lane, rem, h, c);
    }
}

// The sum of squares of the gradients of a CTA's share of the units (an even run of them), in 64 bits from a thread's
// share of one unit on.
template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads) k_grad_squares(const __grid_constant__ Table<CAP> tab, double *__restrict__ part)
{
    __shared__ double sums[kWarps];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t units = tab.first[tab.count];
    uint32_t u = (uint32_t)(units * blockIdx.x / gridDim.x);
    const uint32_t end = (uint32_t)(units * (blockIdx.x + 1) / gridDim.x);
    double sum = 0.0;
    int i = tensor_of(tab, u);
    for (; u < end; ++u) {
        while (u >= tab.first[i + 1]) ++i;
        const int64_t n = tab.n[i];
        const bool vec = (tab.vec[i >> 5] >> (i & 31)) & 1u;
        const G *const g = static_cast<const G *>(tab.g[i]);
        int64_t b = (int64_t)(u - tab.first[i]) * tab.passes * kWarps + warp;
        float s = 0.0f;
        for (int p = 0; p < tab.passes; ++p, b += kWarps) {
            const int64_t at = b * kBlock;
            if (at >= n) break;
            const int rem = n - at < kBlock ? (int)(n - at) : kBlock;
            float x[8];
            if (vec && rem == kBlock) load8<true>(g + at, lane, rem, x);
            else load8<false>(g + at, lane, rem, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], s);
        }
        sum += (double)s;
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kWarps; ++k) sum += sums[k];
        part[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(kThreads) k_grad_norm(const double *__restrict__ part, int64_t parts, float max_norm, float *__restrict__ out)
{
    __shared__ double sums[kWarps];
    griddep_wait();
    griddep_launch_dependents();
    double sum = 0.0;
    for (int64_t k = threadIdx.x; k < parts; k += kThreads) sum += part[k];
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kWarps; ++k) sum += sums[k];
        const float norm = (float)sqrt(sum);
        out[0] = norm;
        out[1] = !isfinite(norm) ? __int_as_float(0x7fffffff) : max_norm > 0.0f ? fminf(1.0f, max_norm / (norm + 1e-6f)) : 1.0f;
    }
}

// ---- plans --------------------------------------------------------------------------------------
const Plan *plan_of(const void *p)
{
    const Plan *plan = static_cast<const Plan *>(p);
    if (!plan || reinterpret_cast<uintptr_t>(p) % 8 || plan->magic != kMagic) return nullptr;
    return plan;
}
size_t table_bytes(const Plan &p) { return p.small ? sizeof(Table<kSmall>) : sizeof(Table<kLarge>); }
const void *table_at(const Plan &p, int64_t k)
{
    return reinterpret_cast<const char *>(&p + 1) + (size_t)k * table_bytes(p);
}
template <int CAP> uint32_t units_of(const void *t)
{
    const Table<CAP> &tab = *static_cast<const Table<CAP> *>(t);
    return tab.first[tab.count];
}
uint32_t units_at(const Plan &p, int64_t k)
{
    return p.small ? units_of<kSmall>(table_at(p, k)) : units_of<kLarge>(table_at(p, k));
}

struct Span {
    uintptr_t lo, hi;
    bool out;
};
int64_t tables_for(int64_t count) { return (count + kLarge - 1) / kLarge; }
size_t plan_size(int64_t count)
{
    const size_t tables = count <= kSmall ? sizeof(Table<kSmall>) : (size_t)tables_for(count) * sizeof(Table<kLarge>);
    return sizeof(Plan) + tables + (size_t)count * 7 * sizeof(Span);   // (the spans: scratch of the overlap check)
}
bool count_ok(int64_t count) { return count >= 0 && count <= (int64_t(1) << 24); }

// Fills the tables with the tensors that have elements. passes: the blocks that a warp takes one after the other.
template <int CAP> int64_t lay_out(const resbm_adamw_desc &d, const resbm_adamw_tensor *tensors, int64_t count, int passes, Table<CAP> *tabs)
{
    const size_t ws = d.w_dtype == RESBM_BF16 ? 2 : 4, gs = d.g_dtype == RESBM_BF16 ? 2 : 4;
    const size_t ss = d.state == RESBM_STATE_E4M3 ? 1 : 4;
    Table<CAP> *t = nullptr;
    int64_t tables = 0;
    for (int64_t i = 0; i < count; ++i) {
        const resbm_adamw_tensor &x = tensors[i];
        if (x.n == 0) continue;
        if (!t || t->count == CAP) {
            t = tabs + tables++;
            memset(t, 0, sizeof *t);
            t->passes = passes;
        }
        const int k = t->count++;
        t->g[k] = x.g;
        t->n[k] = x.n;
        bool vec = ptr_ok(x.g, 4 * gs, true);
        if (d.state != RESBM_STATE_NONE) {
            t->w[k] = x.w;
            t->m[k] = x.m;
            t->v[k] = x.v;
            t->ms[k] = x.m_scale;
            t->vs[k] = x.v_scale;
            t->master[k] = x.master;
            vec = vec && ptr_ok(x.w, 4 * ws, true) && ptr_ok(x.m, 4 * ss, true) && ptr_ok(x.v, 4 * ss, true) && ptr_ok(x.master, 16, false);
        }
        if (vec) t->vec[k >> 5] |= 1u << (k & 31);
        const int64_t per = (int64_t)passes * kWarps * kBlock;
        t->first[k + 1] = t->first[k] + (uint32_t)((x.n + per - 1) / per);
    }
    return tables;
}

resbm_status launch_table(const void *kernel, const Plan &p, int64_t k, unsigned grid, void *second, const Ctx &c)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = c.stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {const_cast<void *>(table_at(p, k)), second};
    const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return cuda_fail(e);
    }
    count_launches(1);
    return RESBM_OK;
}

template <typename W, typename G, bool MASTER> const void *adamw_kernel(const Plan &p)
{
    if (p.state == RESBM_STATE_E4M3)
        return p.small ? (const void *)k_adamw<W, G, MASTER, 8, kSmall> : (const void *)k_adamw<W, G, MASTER, 8, kLarge>;
    return p.small ? (const void *)k_adamw<W, G, MASTER, 32, kSmall> : (const void *)k_adamw<W, G, MASTER, 32, kLarge>;
}
template <typename G> const void *adamw_kernel(const Plan &p)
{
    using bf = __nv_bfloat16;
    return p.w_dtype == RESBM_F32 ? adamw_kernel<float, G, false>(p) : p.master ? adamw_kernel<bf, G, true>(p) : adamw_kernel<bf, G, false>(p);
}
template <typename G> const void *squares_kernel(const Plan &p)
{
    return p.small ? (const void *)k_grad_squares<G, kSmall> : (const void *)k_grad_squares<G, kLarge>;
}

bool dtype_ok(int32_t t) { return t == RESBM_F32 || t == RESBM_BF16; }
bool finite_nonneg(double x) { return x >= 0.0 && x < HUGE_VAL; }

unsigned norm_grid(const Plan &p, int64_t k) { return std::min<unsigned>(units_at(p, k), kNormGrid); }
// The partial sums of `count` plans, or -1 where one of them is none
int64_t norm_parts(const void *const *plans, int64_t count)
{
    if (count < 0 || (count > 0 && !plans)) return -1;
    int64_t parts = 0;
    for (int64_t i = 0; i < count; ++i) {
        const Plan *p = plan_of(plans[i]);
        if (!p) return -1;
        for (int64_t k = 0; k < p->tables; ++k) parts += norm_grid(*p, k);
    }
    return parts;
}

}  // namespace
}  // namespace resbm

using namespace resbm;

extern "C" {

resbm_status resbm_adamw_plan_bytes(int64_t count, size_t *bytes)
{
    if (!bytes || !count_ok(count)) return RESBM_ERR_INVALID_ARG;
    *bytes = plan_size(count);
    return RESBM_OK;
}

resbm_status resbm_adamw_plan(const resbm_adamw_desc *desc, const resbm_adamw_tensor *tensors, int64_t count, void *plan, size_t plan_bytes)
{
    if (!desc || !count_ok(count) || (count > 0 && !tensors)) return RESBM_ERR_INVALID_ARG;
    const resbm_adamw_desc d = *desc;
    const bool states = d.state != RESBM_STATE_NONE, coded = d.state == RESBM_STATE_E4M3;
    if (!dtype_ok(d.w_dtype) || !dtype_ok(d.g_dtype) || d.flags || (states && !coded && d.state != RESBM_STATE_F32)) return RESBM_ERR_INVALID_ARG;
    if (!plan || reinterpret_cast<uintptr_t>(plan) % 8) return RESBM_ERR_INVALID_ARG;
    if (plan_bytes < plan_size(count)) return RESBM_ERR_WORKSPACE;
    const size_t ws = d.w_dtype == RESBM_BF16 ? 2 : 4, gs = d.g_dtype == RESBM_BF16 ? 2 : 4, ss = coded ? 1 : 4;
    // every tensor by itself, and its spans of memory for the check against the others
    Plan *const out = static_cast<Plan *>(plan);
    out->magic = 0;
    Span *const spans = reinterpret_cast<Span *>(static_cast<char *>(plan) + plan_size(count) - (size_t)count * 7 * sizeof(Span));
    int64_t ns = 0, total = 0, masters = 0, filled = 0;
    for (int64_t i = 0; i < count; ++i) {
        const resbm_adamw_tensor &x = tensors[i];
        if (x.n < 0) return RESBM_ERR_INVALID_ARG;
        if (x.n > (int64_t(1) << 40) - total) return RESBM_ERR_UNSUPPORTED;
        if (x.n == 0) continue;
        total += x.n;
        ++filled;
        if (!ptr_ok(x.g, gs, true)) return RESBM_ERR_INVALID_ARG;
        auto add = [&](const void *p, int64_t n, size_t es, bool o) {
            const Range r = rng(p, n, es);
            spans[ns++] = Span{r.lo, r.hi, o};
        };
        add(x.g, x.n, gs, false);
        if (!states) continue;
        if (!ptr_ok(x.w, ws, true) || !ptr_ok(x.m, ss, true) || !ptr_ok(x.v, ss, true) || !ptr_ok(x.master, 4, false)) return RESBM_ERR_INVALID_ARG;
        if (!ptr_ok(x.m_scale, 4, coded) || !ptr_ok(x.v_scale, 4, coded) || (!coded && (x.m_scale || x.v_scale))) return RESBM_ERR_INVALID_ARG;
        if (x.master && d.w_dtype != RESBM_BF16) return RESBM_ERR_INVALID_ARG;
        add(x.w, x.n, ws, true);
        add(x.m, x.n, ss, true);
        add(x.v, x.n, ss, true);
        if (x.master) {
            add(x.master, x.n, 4, true);
            ++masters;
        }
        if (coded) {
            const int64_t blocks = (x.n + kBlock - 1) / kBlock;
            add(x.m_scale, blocks, 4, true);
            add(x.v_scale, blocks, 4, true);
        }
    }
    if (masters && masters != filled) return RESBM_ERR_INVALID_ARG;
    std::sort(spans, spans + ns, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    uintptr_t out_hi = 0, in_hi = 0;   // how far what was written, and read, reaches so far
    for (int64_t k = 0; k < ns; ++k) {
        if (spans[k].lo < out_hi || (spans[k].out && spans[k].lo < in_hi)) return RESBM_ERR_INVALID_ARG;
        uintptr_t &hi = spans[k].out ? out_hi : in_hi;
        hi = std::max(hi, spans[k].hi);
    }
    out->small = count <= kSmall;
    out->w_dtype = d.w_dtype;
    out->g_dtype = d.g_dtype;
    out->state = d.state;
    out->master = masters > 0;
    out->pad = 0;
    const int passes = 1;
    out->tables = out->small ? lay_out(d, tensors, count, passes, reinterpret_cast<Table<kSmall> *>(out + 1))
                             : lay_out(d, tensors, count, passes, reinterpret_cast<Table<kLarge> *>(out + 1));
    out->magic = kMagic;
    return RESBM_OK;
}

resbm_status resbm_adamw_step(const void *plan, const resbm_adamw_hyper *hyper, void *stream)
{
    const Plan *p = plan_of(plan);
    if (!p || !hyper || p->state == RESBM_STATE_NONE) return RESBM_ERR_INVALID_ARG;
    const resbm_adamw_hyper &a = *hyper;
    if (!finite_nonneg(a.lr) || !finite_nonneg(a.eps) || !finite_nonneg(a.weight_decay) || !(a.beta1 >= 0.0 && a.beta1 < 1.0) ||
        !(a.beta2 >= 0.0 && a.beta2 < 1.0) || (!a.step_dev && a.step < 1) || !ptr_ok(a.lr_dev, 4, false) ||
        !ptr_ok(a.step_dev, 8, false) || !ptr_ok(a.grad_scale, 4, false))
        return RESBM_ERR_INVALID_ARG;
    Ctx c;
    resbm_status s = make_ctx(stream, &c);
    Step h = {};
    const double t = a.step_dev ? 1.0 : (double)a.step;
    h.b1 = (float)a.beta1;
    h.omb1 = (float)(1.0 - a.beta1);
    h.b2 = (float)a.beta2;
    h.omb2 = (float)(1.0 - a.beta2);
    h.lnb1 = (float)log(a.beta1);   // (beta = 0: minus infinity, 1 - beta^t = 1)
    h.lnb2 = (float)log(a.beta2);
    h.step_size = (float)(a.lr / -expm1(t * log(a.beta1)));
    h.root = (float)(1.0 / sqrt(-expm1(t * log(a.beta2))));
    h.eps = (float)a.eps;
    h.decay = (float)(1.0 - a.lr * a.weight_decay);
    h.lr = (float)a.lr;
    h.wd = (float)a.weight_decay;
    h.t = (float)t;
    h.lr_dev = a.lr_dev;
    h.step_dev = a.step_dev;
    h.grad_scale = a.grad_scale;
    const void *kernel = p->g_dtype == RESBM_F32 ? adamw_kernel<float>(*p) : adamw_kernel<__nv_bfloat16>(*p);
    for (int64_t k = 0; s == RESBM_OK && k < p->tables; ++k) s = launch_table(kernel, *p, k, units_at(*p, k), &h, c);
    return s;
}

resbm_status resbm_grad_norm_workspace_bytes(const void *const *plans, int64_t count, size_t *bytes)
{
    const int64_t parts = norm_parts(plans, count);
    if (parts < 0 || !bytes) return RESBM_ERR_INVALID_ARG;
    *bytes = (size_t)parts * sizeof(double);
    return RESBM_OK;
}

resbm_status resbm_grad_norm(const void *const *plans, int64_t count, float max_norm, float *out, void *ws, size_t ws_bytes, void *stream)
{
    const int64_t parts = norm_parts(plans, count);
    if (parts < 0 || !(max_norm >= 0.0f) || !(max_norm < INFINITY) || !ptr_ok(out, 4, true)) return RESBM_ERR_INVALID_ARG;
    const size_t need = (size_t)parts * sizeof(double);
    if (need && (!ws || ws_bytes < need)) return RESBM_ERR_WORKSPACE;
    if (need && reinterpret_cast<uintptr_t>(ws) % 256) return RESBM_ERR_INVALID_ARG;
    if (overlaps(rng(out, 2, 4), rng(ws, (int64_t)need, 1))) return RESBM_ERR_INVALID_ARG;
    Ctx c;
    resbm_status s = make_ctx(stream, &c);
    double *part = static_cast<double *>(ws);
    for (int64_t i = 0; s == RESBM_OK && i < count; ++i) {
        const Plan &p = *plan_of(plans[i]);
        const void *kernel = p.g_dtype == RESBM_F32 ? squares_kernel<float>(p) : squares_kernel<__nv_bfloat16>(p);
        for (int64_t k = 0; s == RESBM_OK && k < p.tables; ++k) {
            const unsigned grid = norm_grid(p, k);
            s = launch_table(kernel, p, k, grid, &part, c);
            part += grid;
        }
    }
    if (s != RESBM_OK) return s;
    const cudaError_t e = launch_pdl(k_grad_norm, dim3(1), dim3(kThreads), 0, c, static_cast<const double *>(ws), parts, max_norm, out);
    if (e == cudaSuccess) count_launches(1);
    return finish(e);
}

}  // extern "C"
