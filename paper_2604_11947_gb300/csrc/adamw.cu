// adamw.cu -- resbm_adamw_step and resbm_grad_norm: one pass over many tensors a launch (include/resbm_train.h).
//
// Both are bound by memory: a step with 32-bit states moves 22 bytes an element (bf16 weight and gradient), one
// with 8-bit states 10, the norm 2. The list of tensors travels as the launch's parameter (up to 448 tensors, 31 KB), so
// that nothing is copied to the device and a captured launch carries its own list; a list of up to 32 takes the small
// parameter (2.2 KB; one call on the host 5.1 us, 5.5 with the large one). 308 M bf16 parameters on a GB300: 32-bit states
// 963 us (7.0 TB/s; a copy moves 6.8), 8-bit states 459 (6.8 TB/s), norm 92 (6.7 TB/s).
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "abi.h"
#include "common.cuh"
#include "fp8.cuh"
#include "pair.cuh"
#include "resbm_train.h"

namespace resbm {
namespace {

// CTAs of 128 threads, eight on an SM: with 256 threads the 8-bit step takes 471 us instead of 460, the norm 94 instead of 92.
constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kBlock = RESBM_STATE_BLOCK;             // elements a warp takes at a time: one block of 8-bit states
// Blocks that a warp has in flight where its accesses are vectors, by the states' bits. 8: 308 M elements 564 us with one
// and 461 with two (at 64 registers, some of them spilled: 510 at 72 without spills, with one CTA fewer on an SM; three
// 566). 32: 1058 us either way with the norm, and small lists spread over more CTAs with one.
__host__ __device__ constexpr int deep_of(int bits) { return bits == 8 ? 2 : 1; }
constexpr int kSmall = 32, kLarge = 448;              // tensors a launch, by the parameter's size
constexpr int kNormGrid = 1216;                       // most CTAs of the gradients' norm: eight on each of 152 SMs
// Gradients for a CTA of the norm to be worth it, two rounds of loads in bf16: 10.5 M gradients 1.6 us less than with half as
// many, 1.4 than with four times
constexpr int kRound = 16384;
constexpr float kLeastNormal = 0x1p-126f, kLeastRoot = 0x1p-63f;   // (the second its root)
constexpr uint64_t kMagic = 0x7265736264616d77ull;

// The tensors of one launch, of one kind: those whose accesses are vectors (everything of a tensor aligned to eight
// elements) and the others, whose single elements need fewer registers and one block a warp (30 M elements one past
// alignment, 8-bit states: 98 us; 214 in the vectors' kernel at its registers). A unit is what one CTA takes:
// kWarps * deep blocks of one tensor.
template <int CAP> struct Table {
    void *w[CAP];
    const void *g[CAP];
    void *m[CAP], *v[CAP];
    float *ms[CAP], *vs[CAP];
    float *master[CAP];
    int64_t n[CAP];
    uint32_t first[CAP + 1];      // a tensor's first unit; first[count]: all units
    int32_t count, vec, deep, pad;

    __host__ __device__ int64_t unit() const { return (int64_t)kWarps * kBlock * deep; }   // elements
};
static_assert(sizeof(Table<kLarge>) <= 32000, "the launch's parameters are at most 32764 bytes");

struct Plan {
    uint64_t magic;
    int64_t tables;               // Table<kSmall> if small, else Table<kLarge>, one after the other behind this
    int32_t small, w_dtype, g_dtype, state, master;
    int32_t most;                 // tables that the list can need, however its tensors are aligned
};
static_assert(sizeof(Plan) % 8 == 0, "tables start aligned");

struct Step {
    float b1, omb1, b2, omb2;     // beta and 1 - beta
    float step_size;              // lr / (1 - beta1^t)
    float root;                   // 1 / sqrt(1 - beta2^t)
    float eps, decay;             // decay: 1 - lr weight_decay
    float least;                  // the smallest denominator: of v = 2^-126, with eps
    float nought;                 // minus zero (alone)
    float lr, wd, lnb1, lnb2, t;  // for the values that the device gives
    const float *lr_dev;
    const int64_t *step_dev;
    const float *grad_scale;
};

// Eight elements of a warp's block: lane l has the neighbours 8 l .. 8 l + 7 in one access of 8, 16 or 32 bytes (kVec), or
// l, l + 32, ... one by one (kSingle), below `rem` (kPart).
enum Mode { kVec, kSingle, kPart };
template <Mode MODE> __device__ __forceinline__ void load8(const float *p, int lane, int rem, float (&x)[8])
{
    if (MODE == kVec) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                     : "l"(p + lane * 8));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = MODE == kSingle || j * 32 + lane < rem ? p[j * 32 + lane] : 0.0f;
    }
}
template <Mode MODE> __device__ __forceinline__ void load8(const __nv_bfloat16 *p, int lane, int rem, float (&x)[8])
{
    if (MODE == kVec) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p + lane * 8);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = MODE == kSingle || j * 32 + lane < rem ? to_f32(p[j * 32 + lane]) : 0.0f;
    }
}
template <Mode MODE> __device__ __forceinline__ void load8(const uint8_t *p, int lane, int rem, float (&x)[8])
{
    if (MODE == kVec) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p + lane * 8);
        const float4 a = from_e4m3x4(u.x), b = from_e4m3x4(u.y);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = MODE == kSingle || j * 32 + lane < rem ? from_e4m3(p[j * 32 + lane]) : 0.0f;
    }
}
template <Mode MODE> __device__ __forceinline__ void store8(float *p, int lane, int rem, const float (&x)[8])
{
    if (MODE == kVec) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + lane * 8), "f"(x[0]), "f"(x[1]), "f"(x[2]),
                     "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                     : "memory");
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (MODE == kSingle || j * 32 + lane < rem) p[j * 32 + lane] = x[j];
    }
}
template <Mode MODE> __device__ __forceinline__ void store8(__nv_bfloat16 *p, int lane, int rem, const float (&x)[8])
{
    if (MODE == kVec) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p + lane * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (MODE == kSingle || j * 32 + lane < rem) p[j * 32 + lane] = from_f32<__nv_bfloat16>(x[j]);
    }
}
// (values in units of their scale)
template <Mode MODE> __device__ __forceinline__ void store8(uint8_t *p, int lane, int rem, const float (&x)[8])
{
    if (MODE == kVec) {
        *reinterpret_cast<uint2 *>(p + lane * 8) = make_uint2(e4m3x4(x[0], x[1], x[2], x[3]), e4m3x4(x[4], x[5], x[6], x[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (MODE == kSingle || j * 32 + lane < rem) p[j * 32 + lane] = e4m3x1(x[j]);
    }
}

// Root and reciprocal by the approximate instructions (errors under 2^-22), which take normal numbers only
__device__ __forceinline__ float approx_sqrt(float v)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float approx_rsqrt(float v)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float approx_rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Two roots to nearest, for the roots that are stored: an 8-bit code next to a border takes the other side with the last bit of
// what it is made from. From an approximate reciprocal root y, r = v y and the remainder v - r^2 (exact as a fused
// multiply-add), one step of Newton's method (Markstein, "Computation of elementary functions on the IBM RISC System/6000
// processor", 1990): r + (v - r^2) y / 2. Compared with __fsqrt_rn for every float: equal from 2^-102 on, where the
// remainder is no denormal yet, below within a bit; from 2^-126 down 2^63 v or less, but above zero where v is. Infinity
// gives a NaN (a choice of infinity costs 45 us, at 64 registers a thread). The 8-bit step of 308 M elements takes 459 us
// with it, 541 with __fsqrt_rn, 447 with approximate roots, of which one in six is a bit off.
__device__ __forceinline__ void roots(Pair v, float &r0, float &r1)
{
    float v0, v1;
    split(v, v0, v1);
    const Pair y = pair(approx_rsqrt(fmaxf(v0, kLeastNormal)), approx_rsqrt(fmaxf(v1, kLeastNormal))), r = v * y;
    split(r, r0, r1);
    split(fma(pair(fmaf(-r0, r0, v0), fmaf(-r1, r1, v1)), y * both(0.5f), r), r0, r1);
}

// A product that is rounded by itself although a sum follows. Left as a product the compiler makes one fused
// multiply-add of it and the sum, whatever rounding the two were written with; what this one adds is minus zero, which
// leaves every value as it is, and which the compiler does not know.
__device__ __forceinline__ Pair alone(Pair a, Pair b, const Step &h) { return fma(a, b, both(h.nought)); }

// K blocks of 256 elements by one warp, kWarps blocks apart (or one, the last `rem` of a tensor). The products of the
// running means are rounded one by one (alone): a fused multiply-add would move values next to a rounding border of e4m3
// across it, and the same step would then depend on the compiler's contractions; so would an approximate sqrt(v) where it is
// stored (roots). The quotient m / (sqrt(v) ..) is approximate, far below what the update is to the weight, and so is
// the root with 32-bit states. A v below 2^-126 (gradients below 1e-17) counts as that for the weight (`least` is its
// denominator).
// The 8-bit form is bound by instructions as much as by memory (10 bytes an element): with IEEE roots and quotients, one
// value an instruction and one block a warp 75 of them an element, 868 us for 308 M elements; with pairs, two blocks a warp,
// accesses of eight elements, approximate quotients and one reciprocal an element, and roots() 40 and 459.
template <typename W, typename G, bool MASTER, int BITS, Mode MODE, int K>
__device__ __forceinline__ void adamw_blocks(W *w, const G *g, void *mp, void *vp, float *ms, float *vs, float *master,
                                             int lane, int rem, const Step &h, float c)
{
    using S = typename std::conditional<BITS == 8, uint8_t, float>::type;
    constexpr int kNext = kWarps * kBlock;
    S *const m8 = static_cast<S *>(mp), *const v8 = static_cast<S *>(vp);
    float x[K][8], dg[K][8], m[K][8], v[K][8];
    float sm[K], sv[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (BITS == 8) {
            sm[k] = ms[k * kWarps];
            sv[k] = vs[k * kWarps];
        }
        load8<MODE>(static_cast<const S *>(m8 + k * kNext), lane, rem, m[k]);
        load8<MODE>(static_cast<const S *>(v8 + k * kNext), lane, rem, v[k]);
        load8<MODE>(g + k * kNext, lane, rem, dg[k]);
        if (MASTER) load8<MODE>(static_cast<const float *>(master + k * kNext), lane, rem, x[k]);
        else load8<MODE>(static_cast<const W *>(w + k * kNext), lane, rem, x[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float am = 0.0f, av = 0.0f;   // the largest |m| and sqrt(v)
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const Pair g2 = pair(dg[k][j], dg[k][j + 1]) * both(c);
            Pair m2 = pair(m[k][j], m[k][j + 1]), v2 = pair(v[k][j], v[k][j + 1]);
            if (BITS == 8) {
                m2 = m2 * both(sm[k]);
                v2 = v2 * both(sv[k]);
                v2 = v2 * v2;
            }
            m2 = alone(m2, both(h.b1), h) + alone(g2, both(h.omb1), h);
            v2 = alone(v2, both(h.b2), h) + alone(g2 * g2, both(h.omb2), h);
            float m0, m1, v0, v1, d0, d1;
            split(m2, m0, m1);
            split(v2, v0, v1);
            float r0, r1;
            if (BITS == 8) {
                roots(v2, r0, r1);
            } else {
                r0 = approx_sqrt(v0);
                r1 = approx_sqrt(v1);
            }
            split(fma(pair(r0, r1), both(h.root), both(h.eps)), d0, d1);
            const Pair q = m2 * pair(approx_rcp(max_nan(d0, h.least)), approx_rcp(max_nan(d1, h.least)));
            split(fma(q, both(-h.step_size), pair(x[k][j], x[k][j + 1]) * both(h.decay)), x[k][j], x[k][j + 1]);
            m[k][j] = m0;
            m[k][j + 1] = m1;
            v[k][j] = BITS == 8 ? r0 : v0;
            v[k][j + 1] = BITS == 8 ? r1 : v1;
            if (BITS == 8) {
                am = max_nan(am, max_nan(fabsf(m0), fabsf(m1)));
                av = max_nan(av, max_nan(r0, r1));
            }
        }
        if (MASTER) store8<MODE>(master + k * kNext, lane, rem, x[k]);
        store8<MODE>(w + k * kNext, lane, rem, x[k]);
        if (BITS == 8) {
            const E4m3Scale a = e4m3_scale(__reduce_max_sync(0xffffffffu, abs_bits(am))), b = e4m3_scale(__reduce_max_sync(0xffffffffu, abs_bits(av)));
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                // a sqrt(v) above zero (at least 2^-87 then) keeps a code above zero
                float l0, l1;
                split(pair(v[k][j], v[k][j + 1]) * both(0x1p78f), l0, l1);
                split(pair(m[k][j], m[k][j + 1]) * both(a.inv), m[k][j], m[k][j + 1]);
                split(pair(v[k][j], v[k][j + 1]) * both(b.inv), v[k][j], v[k][j + 1]);
                v[k][j] = max_nan(v[k][j], fminf(l0, kE4m3Least));
                v[k][j + 1] = max_nan(v[k][j + 1], fminf(l1, kE4m3Least));
            }
            if (lane == 0) {
                ms[k * kWarps] = a.scale;
                vs[k * kWarps] = b.scale;
            }
        }
        store8<MODE>(m8 + k * kNext, lane, rem, m[k]);
        store8<MODE>(v8 + k * kNext, lane, rem, v[k]);
    }
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

template <typename W, typename G, bool MASTER, int BITS, bool VEC, int CAP>
__global__ void __launch_bounds__(kThreads, VEC && BITS == 8 ? 8 : 1) k_adamw(const __grid_constant__ Table<CAP> tab, const __grid_constant__ Step given)
{
    Step h = given;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = tensor_of(tab, blockIdx.x);
    const int64_t n = tab.n[i];
    int64_t b = (int64_t)(blockIdx.x - tab.first[i]) * tab.deep * kWarps + warp;
    griddep_wait();
    griddep_launch_dependents();
    float c = 1.0f;
    if (h.grad_scale) {
        c = *h.grad_scale;
        if (!isfinite(c)) return;
    }
    if (h.lr_dev || h.step_dev) {
        const float lr = h.lr_dev ? *h.lr_dev : h.lr;
        const float t = h.step_dev ? fmaxf((float)*h.step_dev, 1.0f) : h.t;
        h.step_size = lr / -expm1f(t * h.lnb1);
        h.root = 1.0f / sqrtf(-expm1f(t * h.lnb2));
        h.decay = 1.0f - lr * h.wd;
        h.least = fmaf(h.root, kLeastRoot, h.eps);
    }
    W *const w = static_cast<W *>(tab.w[i]);
    const G *const g = static_cast<const G *>(tab.g[i]);
    char *const m = static_cast<char *>(tab.m[i]), *const v = static_cast<char *>(tab.v[i]);
    float *const ms = tab.ms[i], *const vs = tab.vs[i], *const master = tab.master[i];
    constexpr int ss = BITS / 8, K = VEC ? deep_of(BITS) : 1;
    auto run = [&](auto mode, auto deep, int rem) {
        const int64_t at = b * kBlock;
        adamw_blocks<W, G, MASTER, BITS, (Mode)decltype(mode)::value, decltype(deep)::value>(
            w + at, g + at, m + at * ss, v + at * ss, ms + b, vs + b, master + at, lane, rem, h, c);
    };
    using std::integral_constant;
    if (b * kBlock + ((K - 1) * kWarps + 1) * kBlock <= n) {
        run(integral_constant<int, VEC ? kVec : kSingle>(), integral_constant<int, K>(), kBlock);
        return;
    }
    for (int k = 0; k < K; ++k, b += kWarps) {   // the end of a tensor
        const int64_t rem = n - b * kBlock;
        if (rem <= 0) return;
        if (VEC && rem >= kBlock) run(integral_constant<int, kVec>(), integral_constant<int, 1>(), kBlock);
        else run(integral_constant<int, kPart>(), integral_constant<int, 1>(), (int)min(rem, (int64_t)kBlock));
    }
}

// Sum of squares of g[from .. to) by a CTA, this thread's share: 16-byte loads, eight in flight, from the first element on
// whose address is a multiple of 16; in 64 bits from one round of loads on.
template <typename G> __device__ __forceinline__ double squares(const G *g, int64_t from, int64_t to)
{
    constexpr int V = 16 / (int)sizeof(G), kDeep = 8;
    double sum = 0.0;
    const int64_t head = min(to, from + (int64_t)((16 - reinterpret_cast<uintptr_t>(g + from) % 16) % 16 / sizeof(G)));
    const int64_t vectors = (to - head) / V;
    const uint4 *const p = reinterpret_cast<const uint4 *>(g + head);
    auto add = [](uint4 u, float &s) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(G) == 2) {
                const float a = __uint_as_float(w[i] << 16), b = __uint_as_float(w[i] & 0xFFFF0000u);
                s = fmaf(a, a, s);
                s = fmaf(b, b, s);
            } else {
                const float a = __uint_as_float(w[i]);
                s = fmaf(a, a, s);
            }
        }
    };
    int64_t k = threadIdx.x;
    for (; k + (kDeep - 1) * kThreads < vectors; k += kDeep * kThreads) {
        uint4 u[kDeep];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kDeep; ++j) u[j] = p[k + j * kThreads];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) add(u[j], s[j & 1]);
        sum += (double)(s[0] + s[1]);
    }
    float s = 0.0f;
    if (k < vectors) {
        uint4 u[kDeep];
        float a[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kDeep; ++j) u[j] = k + j * kThreads < vectors ? p[k + j * kThreads] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < kDeep; ++j) add(u[j], a[j & 1]);
        sum += (double)(a[0] + a[1]);
    }
    // the elements before the first vector and behind the last
    if (from + threadIdx.x < head) {
        const float a = to_f32(g[from + threadIdx.x]);
        s = fmaf(a, a, s);
    }
    const int64_t tail = head + vectors * V + threadIdx.x;
    if (tail < to) {
        const float a = to_f32(g[tail]);
        s = fmaf(a, a, s);
    }
    return sum + (double)s;
}

// The sum of squares of the gradients of a CTA's share of the units, an even run of them: what it has of each tensor is
// one contiguous piece.
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
    const int64_t per = tab.unit();
    double sum = 0.0;
    for (int i = tensor_of(tab, u); u < end; ++i) {
        const uint32_t stop = min(end, tab.first[i + 1]);
        sum += squares(static_cast<const G *>(tab.g[i]), (int64_t)(u - tab.first[i]) * per, min((int64_t)(stop - tab.first[i]) * per, tab.n[i]));
        u = stop;
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kWarps; ++k) sum += sums[k];
        part[blockIdx.x] = sum;
    }
}

// The partial sums in 64 bits. FP64 adds are slow here, so that a CTA of 256 threads with its loads in one round and its
// warps' sums through another tree takes 4 us less than one of 1024 whose first thread adds them up (308 M gradients 96 -> 92 us,
// 10.5 M 10.5 -> 8.4 with the host's 7.1); 512 threads 92.8, 128 92.1.
constexpr int kNormThreads = 256;
__global__ void __launch_bounds__(kNormThreads) k_grad_norm(const double *__restrict__ part, int64_t parts, float max_norm, float *__restrict__ out)
{
    constexpr int kW = kNormThreads / 32, kDeep = 5;   // (a full grid's partial sums in one round of loads)
    __shared__ double sums[kW];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    for (int64_t k = threadIdx.x; k < parts; k += kDeep * kNormThreads) {
        double x[kDeep];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) x[j] = k + j * kNormThreads < parts ? part[k + j * kNormThreads] : 0.0;
#pragma unroll
        for (int j = 0; j < kDeep; ++j) sum += x[j];
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {
        sum = lane < kW ? sums[lane] : 0.0;
        for (int o = kW / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) {
            const float norm = (float)sqrt(sum);
            out[0] = norm;
            out[1] = !isfinite(norm) ? __int_as_float(0x7fffffff) : max_norm > 0.0f ? fminf(1.0f, max_norm / (norm + 1e-6f)) : 1.0f;
        }
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
struct Extent {
    uint32_t units;
    int64_t unit;   // elements
    bool vec;
};
template <int CAP> Extent extent_of(const void *t)
{
    const Table<CAP> &tab = *static_cast<const Table<CAP> *>(t);
    return {tab.first[tab.count], tab.unit(), tab.vec != 0};
}
Extent extent_at(const Plan &p, int64_t k)
{
    return p.small ? extent_of<kSmall>(table_at(p, k)) : extent_of<kLarge>(table_at(p, k));
}

struct Span {
    uintptr_t lo, hi;
    bool out;
};
// (either kind of tensors may end in a table that is not full)
int64_t most_tables(int64_t count) { return count <= kSmall ? 2 : (count + kLarge - 1) / kLarge + 1; }
size_t plan_size(int64_t count)
{
    const size_t tables = (size_t)most_tables(count) * (count <= kSmall ? sizeof(Table<kSmall>) : sizeof(Table<kLarge>));
    return sizeof(Plan) + tables + (size_t)count * 7 * sizeof(Span);   // (the spans: scratch of the overlap check)
}
bool count_ok(int64_t count) { return count >= 0 && count <= (int64_t(1) << 24); }

// Whether everything of a tensor is aligned to eight elements
bool is_vec(const resbm_adamw_desc &d, const resbm_adamw_tensor &x)
{
    const size_t ws = d.w_dtype == RESBM_BF16 ? 16 : 32, gs = d.g_dtype == RESBM_BF16 ? 16 : 32, ss = d.state == RESBM_STATE_E4M3 ? 8 : 32;
    if (!ptr_ok(x.g, gs, true)) return false;
    return d.state == RESBM_STATE_NONE || (ptr_ok(x.w, ws, true) && ptr_ok(x.m, ss, true) && ptr_ok(x.v, ss, true) && ptr_ok(x.master, 32, false));
}

// Fills the tables with the tensors that have elements, one kind after the other.
template <int CAP> int64_t lay_out(const resbm_adamw_desc &d, const resbm_adamw_tensor *tensors, int64_t count, Table<CAP> *tabs)
{
    int64_t tables = 0;
    for (int vec = 1; vec >= 0; --vec) {
        Table<CAP> *t = nullptr;
        for (int64_t i = 0; i < count; ++i) {
            const resbm_adamw_tensor &x = tensors[i];
            if (x.n == 0 || is_vec(d, x) != (vec != 0)) continue;
            if (!t || t->count == CAP) {
                t = tabs + tables++;
                memset(t, 0, sizeof *t);
                t->vec = vec;
                t->deep = vec && d.state != RESBM_STATE_NONE ? deep_of(d.state) : 1;
            }
            const int k = t->count++;
            t->g[k] = x.g;
            t->n[k] = x.n;
            if (d.state != RESBM_STATE_NONE) {
                t->w[k] = x.w;
                t->m[k] = x.m;
                t->v[k] = x.v;
                t->ms[k] = x.m_scale;
                t->vs[k] = x.v_scale;
                t->master[k] = x.master;
            }
            t->first[k + 1] = t->first[k] + (uint32_t)((x.n + t->unit() - 1) / t->unit());
        }
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

template <typename W, typename G, bool MASTER, int BITS> const void *adamw_kernel(const Plan &p, bool vec)
{
    if (vec) return p.small ? (const void *)k_adamw<W, G, MASTER, BITS, true, kSmall> : (const void *)k_adamw<W, G, MASTER, BITS, true, kLarge>;
    return p.small ? (const void *)k_adamw<W, G, MASTER, BITS, false, kSmall> : (const void *)k_adamw<W, G, MASTER, BITS, false, kLarge>;
}
template <typename W, typename G, bool MASTER> const void *adamw_kernel(const Plan &p, bool vec)
{
    return p.state == RESBM_STATE_E4M3 ? adamw_kernel<W, G, MASTER, 8>(p, vec) : adamw_kernel<W, G, MASTER, 32>(p, vec);
}
template <typename G> const void *adamw_kernel(const Plan &p, bool vec)
{
    using bf = __nv_bfloat16;
    return p.w_dtype == RESBM_F32 ? adamw_kernel<float, G, false>(p, vec)
           : p.master             ? adamw_kernel<bf, G, true>(p, vec)
                                  : adamw_kernel<bf, G, false>(p, vec);
}
template <typename G> const void *squares_kernel(const Plan &p)
{
    return p.small ? (const void *)k_grad_squares<G, kSmall> : (const void *)k_grad_squares<G, kLarge>;
}

bool dtype_ok(int32_t t) { return t == RESBM_F32 || t == RESBM_BF16; }
bool finite_nonneg(double x) { return x >= 0.0 && x < HUGE_VAL; }

// CTAs of the gradients' norm: a round of loads for each, up to kNormGrid
unsigned norm_grid(const Plan &p, int64_t k)
{
    const Extent x = extent_at(p, k);
    return (unsigned)std::min<int64_t>((x.units * x.unit + kRound - 1) / kRound, kNormGrid);
}
// The partial sums of `count` plans, or -1 where one of them is none; most: what they come to at most, however their tensors
// are aligned
int64_t norm_parts(const void *const *plans, int64_t count, bool most)
{
    if (count < 0 || (count > 0 && !plans)) return -1;
    int64_t parts = 0;
    for (int64_t i = 0; i < count; ++i) {
        const Plan *p = plan_of(plans[i]);
        if (!p) return -1;
        if (most) parts += (int64_t)p->most * kNormGrid;
        else
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
    out->most = (int32_t)most_tables(count);
    out->tables = out->small ? lay_out(d, tensors, count, reinterpret_cast<Table<kSmall> *>(out + 1))
                             : lay_out(d, tensors, count, reinterpret_cast<Table<kLarge> *>(out + 1));
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
    h.least = h.root * kLeastRoot + h.eps;
    h.nought = -0.0f;
    h.lr = (float)a.lr;
    h.wd = (float)a.weight_decay;
    h.t = (float)t;
    h.lr_dev = a.lr_dev;
    h.step_dev = a.step_dev;
    h.grad_scale = a.grad_scale;
    for (int64_t k = 0; s == RESBM_OK && k < p->tables; ++k) {
        const Extent x = extent_at(*p, k);
        s = launch_table(p->g_dtype == RESBM_F32 ? adamw_kernel<float>(*p, x.vec) : adamw_kernel<__nv_bfloat16>(*p, x.vec), *p, k, x.units, &h, c);
    }
    return s;
}

resbm_status resbm_grad_norm_workspace_bytes(const void *const *plans, int64_t count, size_t *bytes)
{
    const int64_t parts = norm_parts(plans, count, true);
    if (parts < 0 || !bytes) return RESBM_ERR_INVALID_ARG;
    *bytes = (size_t)parts * sizeof(double);
    return RESBM_OK;
}

resbm_status resbm_grad_norm(const void *const *plans, int64_t count, float max_norm, float *out, void *ws, size_t ws_bytes, void *stream)
{
    const int64_t parts = norm_parts(plans, count, false);
    if (parts < 0 || !(max_norm >= 0.0f) || !(max_norm < INFINITY) || !ptr_ok(out, 4, true)) return RESBM_ERR_INVALID_ARG;
    const size_t need = (size_t)norm_parts(plans, count, true) * sizeof(double);
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
    const cudaError_t e = launch_pdl(k_grad_norm, dim3(1), dim3(kNormThreads), 0, c, static_cast<const double *>(ws), parts, max_norm, out);
    if (e == cudaSuccess) count_launches(1);
    return finish(e);
}

}  // extern "C"
