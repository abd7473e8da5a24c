// add_norm.cu -- resbm_add_rmsnorm_fwd: h = x + a, n = h / sqrt(mean h^2 + eps) * gamma, n in the activations'
// type and / or in e4m3 with scales (include/resbm_train.h).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "abi.h"
#include "common.cuh"
#include "fp8.cuh"
#include "pair.cuh"
#include "resbm_train.h"

namespace resbm {
namespace {

struct NormArgs {
    const void *X, *A, *gamma;
    void *H, *N;
    uint8_t *Q;
    float *S;
    int64_t T, ldx, lda, ldh, ldn, groups;
    int d, group_log;             // columns behind a scale, as a power of two >= 32; 30 (over every d) for the whole row
    float eps, inv_d;
};

template <int V> __device__ __forceinline__ void scale_by(float (&f)[V], float c)
{
    if constexpr (V > 1) {
#pragma unroll
        for (int i = 0; i < V; i += 2) split(pair(f[i], f[i + 1]) * both(c), f[i], f[i + 1]);
    } else {
        f[0] *= c;
    }
}

// V neighbouring elements, as loaded
template <typename E, int V> struct Vec {
    static constexpr int kWords = V * (int)sizeof(E) / 4;   // 4
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const E *p)
    {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ void store(E *p) const { *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
    // elements 2 i and 2 i + 1
    __device__ __forceinline__ Pair get(int i) const
    {
        if constexpr (sizeof(E) == 2) return pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        else return pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    }
    __device__ __forceinline__ void set(int i, Pair f)
    {
        float a, b;
        split(f, a, b);
        if constexpr (sizeof(E) == 2) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            w[2 * i] = __float_as_uint(a);
            w[2 * i + 1] = __float_as_uint(b);
        }
    }
    __device__ __forceinline__ void add(const Vec &o)
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) set(i, get(i) + o.get(i));
    }
    __device__ __forceinline__ float squares() const
    {
        Pair s = both(0.0f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) s = fma(get(i), get(i), s);
        float a, b;
        split(s, a, b);
        return a + b;
    }
    __device__ __forceinline__ void scaled(float c, const Vec &g, float (&f)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) split(get(i) * both(c) * g.get(i), f[2 * i], f[2 * i + 1]);
    }
    __device__ __forceinline__ void put(const float (&f)[V])
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) set(i, pair(f[2 * i], f[2 * i + 1]));
    }
    static __device__ __forceinline__ void codes(uint8_t *q, const float (&f)[V])
    {
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
        else *reinterpret_cast<uint32_t *>(q) = e4m3x4(f[0], f[1], f[2], f[3]);
    }
};
template <typename E> struct Vec<E, 1> {
    E u;
    __device__ __forceinline__ void load(const E *p) { u = *p; }
    __device__ __forceinline__ void zero() { u = from_f32<E>(0.0f); }
    __device__ __forceinline__ void store(E *p) const { *p = u; }
    __device__ __forceinline__ void add(const Vec &o) { u = from_f32<E>(to_f32(u) + to_f32(o.u)); }
    __device__ __forceinline__ float squares() const { return to_f32(u) * to_f32(u); }
    __device__ __forceinline__ void scaled(float c, const Vec &g, float (&f)[1]) const { f[0] = to_f32(u) * c * to_f32(g.u); }
    __device__ __forceinline__ void put(const float (&f)[1]) { u = from_f32<E>(f[0]); }
    static __device__ __forceinline__ void codes(uint8_t *q, const float (&f)[1]) { *q = e4m3x1(f[0]); }
};

// The row in registers: TPR threads a row (a warp of a CTA of eight, or a whole CTA), each with KV vectors of V
// elements, thread q of them owning vectors q, q + TPR, ... X and A are read once, H, N, Q and S written once. The
// sum of squares goes through a fixed shuffle tree and the warps' sums in warp order.
template <typename E, int V, int KV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) k_add_norm(const __grid_constant__ NormArgs p)
{
    constexpr int kThreads = TPR == 32 ? 256 : TPR, kRows = kThreads / TPR, kW = TPR / 32;
    __shared__ float sums[kW];
    __shared__ uint32_t most[KV * kW];   // the largest |n| of every 32 vectors
    using L = Vec<E, V>;
    const int tid = threadIdx.x % TPR, lane = threadIdx.x & 31, warp = tid >> 5;
    const int nv = p.d / V;
    const E *const gamma = static_cast<const E *>(p.gamma);
    griddep_wait();
    griddep_launch_dependents();
    for (int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; t < p.T; t += (int64_t)gridDim.x * kRows) {
        const E *const x = static_cast<const E *>(p.X) + t * p.ldx;
        L h[KV], b[KV];
#pragma unroll
        for (int k = 0; k < KV; ++k) {
            const int q = tid + TPR * k;
            if (q < nv) h[k].load(x + q * V);
            else h[k].zero();
        }
        float s = 0.0f;
        if (p.A) {
            const E *const a = static_cast<const E *>(p.A) + t * p.lda;
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                const int q = tid + TPR * k;
                if (q < nv) b[k].load(a + q * V);
                else b[k].zero();
            }
#pragma unroll
            for (int k = 0; k < KV; ++k) h[k].add(b[k]);
        }
#pragma unroll
        for (int k = 0; k < KV; ++k) s += h[k].squares();   // (of h as stored)
        if (p.H) {
            E *const o = static_cast<E *>(p.H) + t * p.ldh;
#pragma unroll
            for (int k = 0; k < KV; ++k)
                if (tid + TPR * k < nv) h[k].store(o + (tid + TPR * k) * V);
        }
        s *= p.inv_d;   // (a thread's share of the mean: the row's sum itself could leave fp32's range)
        // gamma, on its way while the sums travel
#pragma unroll
        for (int k = 0; k < KV; ++k) {
            const int q = tid + TPR * k;
            if (q < nv) b[k].load(gamma + q * V);
            else b[k].zero();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (kW > 1) {
            if (lane == 0) sums[warp] = s;
            __syncthreads();
            s = 0.0f;
#pragma unroll
            for (int w = 0; w < kW; ++w) s += sums[w];
        }
        const float rstd = 1.0f / sqrtf(s + p.eps);
        float n[KV][V];
#pragma unroll
        for (int k = 0; k < KV; ++k) h[k].scaled(rstd, b[k], n[k]);
        if (p.N) {
            E *const o = static_cast<E *>(p.N) + t * p.ldn;
#pragma unroll
            for (int k = 0; k < KV; ++k)
                if (tid + TPR * k < nv) {
                    L r;
                    r.put(n[k]);
                    r.store(o + (tid + TPR * k) * V);
                }
        }
        if (p.Q) {
            // the largest |n| of a group: over the lanes that share it, then, where a group has more than a warp's
            // vectors, over the 32-vector pieces that the warps left in shared memory (a warp's own in registers)
            const int lanes_log = p.group_log - (V == 8 ? 3 : V == 4 ? 2 : 0);
            uint32_t am[KV];
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                float m = fabsf(n[k][0]);
#pragma unroll
                for (int i = 1; i < V; ++i) m = max_nan(m, fabsf(n[k][i]));
                am[k] = __float_as_uint(m) & 0x7FFFFFFFu;
            }
            if (lanes_log >= 5) {
#pragma unroll
                for (int k = 0; k < KV; ++k) am[k] = __reduce_max_sync(0xffffffffu, am[k]);
                const int pieces_log = lanes_log - 5;
                if (pieces_log > 0) {
                    if (kW > 1) {
                        if (lane == 0)
#pragma unroll
                            for (int k = 0; k < KV; ++k) most[k * kW + warp] = am[k];
                        __syncthreads();
#pragma unroll
                        for (int k = 0; k < KV; ++k) {
                            const int c0 = (k * kW + warp) >> pieces_log << pieces_log, c1 = min(c0 + (1 << pieces_log), KV * kW);
                            for (int c = c0; c < c1; ++c) am[k] = max(am[k], most[c]);
                        }
                    } else {
                        uint32_t all[KV];
#pragma unroll
                        for (int k = 0; k < KV; ++k) {
                            all[k] = am[k];
#pragma unroll
                            for (int j = 0; j < KV; ++j)
                                if (j >> pieces_log == k >> pieces_log) all[k] = max(all[k], am[j]);
                        }
#pragma unroll
                        for (int k = 0; k < KV; ++k) am[k] = all[k];
                    }
                }
            } else {
                for (int o = 1 << lanes_log >> 1; o > 0; o >>= 1)
#pragma unroll
                    for (int k = 0; k < KV; ++k) am[k] = max(am[k], __shfl_xor_sync(0xffffffffu, am[k], o));
            }
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                const int q = tid + TPR * k;
                if (q >= nv) continue;
                const E4m3Scale c = e4m3_scale(am[k]);
                scale_by(n[k], c.inv);
                L::codes(p.Q + t * p.d + q * V, n[k]);
                if ((q & ((1 << lanes_log) - 1)) == 0) p.S[t * p.groups + (q >> lanes_log)] = c.scale;
            }
        }
        if (kW > 1) __syncthreads();   // sums and most are this row's until here
    }
}

// Rows too long for the registers: a CTA reads its row again for the second pass (from H where it is stored, which
// may be X or A; every thread reads back what it wrote itself), and a third time where a scale spans the whole row.
template <typename E> __global__ void __launch_bounds__(1024) k_add_norm_long(const __grid_constant__ NormArgs p)
{
    __shared__ float sums[32];
    __shared__ uint32_t peaks[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const E *const gamma = static_cast<const E *>(p.gamma);
    griddep_wait();
    griddep_launch_dependents();
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        const E *const x = static_cast<const E *>(p.X) + t * p.ldx;
        const E *const a = p.A ? static_cast<const E *>(p.A) + t * p.lda : nullptr;
        E *const ho = p.H ? static_cast<E *>(p.H) + t * p.ldh : nullptr;
        auto sum_at = [&](int64_t j) { return a ? to_f32(from_f32<E>(to_f32(x[j]) + to_f32(a[j]))) : to_f32(x[j]); };
        auto h_at = [&](int64_t j) { return ho ? to_f32(ho[j]) : sum_at(j); };
        float s = 0.0f;
        for (int64_t j = tid; j < p.d; j += 1024) {
            const float f = sum_at(j);
            if (ho) ho[j] = from_f32<E>(f);
            s = fmaf(f * p.inv_d, f, s);
        }
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) sums[warp] = s;
        __syncthreads();
        s = 0.0f;
        for (int w = 0; w < 32; ++w) s += sums[w];
        const float rstd = 1.0f / sqrtf(s + p.eps);
        uint32_t am = 0;
        for (int64_t j = tid; j < p.d; j += 1024) {
            const float n = h_at(j) * rstd * to_f32(gamma[j]);
            if (p.N) static_cast<E *>(p.N)[t * p.ldn + j] = from_f32<E>(n);
            am = max(am, abs_bits(n));
        }
        const int64_t group = int64_t(1) << p.group_log;
        if (p.Q && group > p.d) {   // one scale a row
            am = __reduce_max_sync(0xffffffffu, am);
            if (lane == 0) peaks[warp] = am;
            __syncthreads();
            for (int w = 0; w < 32; ++w) am = max(am, peaks[w]);
            const E4m3Scale c = e4m3_scale(am);
            for (int64_t j = tid; j < p.d; j += 1024)
                p.Q[t * p.d + j] = e4m3x1(h_at(j) * rstd * to_f32(gamma[j]) * c.inv);
            if (tid == 0) p.S[t] = c.scale;
        } else if (p.Q) {             // a warp a group (the other warps' H has to be there)
            __syncthreads();
            for (int64_t g = warp; g < p.groups; g += 32) {
                const int64_t j0 = g * group, j1 = min(j0 + group, (int64_t)p.d);
                uint32_t m = 0;
                for (int64_t j = j0 + lane; j < j1; j += 32) m = max(m, abs_bits(h_at(j) * rstd * to_f32(gamma[j])));
                const E4m3Scale c = e4m3_scale(__reduce_max_sync(0xffffffffu, m));
                for (int64_t j = j0 + lane; j < j1; j += 32)
                    p.Q[t * p.d + j] = e4m3x1(h_at(j) * rstd * to_f32(gamma[j]) * c.inv);
                if (lane == 0) p.S[t * p.groups + g] = c.scale;
            }
        }
        __syncthreads();   // sums and peaks are this row's until here
    }
}

template <typename E, int V, int KV, int TPR> cudaError_t launch(const NormArgs &p, const Ctx &c)
{
    constexpr int kThreads = TPR == 32 ? 256 : TPR, kRows = kThreads / TPR;
    const int64_t want = (p.T + kRows - 1) / kRows;
    const unsigned grid = (unsigned)std::min<int64_t>(want, INT32_MAX);
    return launch_pdl(k_add_norm<E, V, KV, TPR>, dim3(grid), dim3(kThreads), 0, c, p);
}

#ifndef KVV
#define KVV 2
#endif
#ifndef KVS
#define KVS 8
#endif
template <typename E, int V> cudaError_t run(const NormArgs &p, const Ctx &c)
{
    const int64_t nv = p.d / V;
    constexpr int K = V > 1 ? KVV : KVS;
    if (nv <= 32) return launch<E, V, 1, 32>(p, c);
    if (nv <= 64) return launch<E, V, 2, 32>(p, c);
    if (nv <= 128) return launch<E, V, 4, 32>(p, c);
    if (V == 1 && nv <= 256) return launch<E, V, 8, 32>(p, c);
    if (nv <= 64 * K) return launch<E, V, K, 64>(p, c);
    if (nv <= 128 * K) return launch<E, V, K, 128>(p, c);
    if (nv <= 256 * K) return launch<E, V, K, 256>(p, c);
    if (nv <= 512 * K) return launch<E, V, K, 512>(p, c);
    if (nv <= 1024 * K) return launch<E, V, K, 1024>(p, c);
    if (nv <= 1024 * 4) return launch<E, V, 4, 1024>(p, c);
    const unsigned grid = (unsigned)std::min<int64_t>(p.T, (int64_t)c.sm_count * 2);
    return launch_pdl(k_add_norm_long<E>, dim3(grid), dim3(1024), 0, c, p);
}

template <typename E> cudaError_t run(const NormArgs &p, const Ctx &c)
{
    // 16-byte vectors where every row of every tensor starts at a multiple of 16 bytes (Q: of the vector's codes)
    constexpr int V = 16 / (int)sizeof(E);
    auto al = [](const void *q, int64_t ld) { return !q || (reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % V == 0); };
    const bool vec = p.d % V == 0 && al(p.X, p.ldx) && al(p.A, p.lda) && al(p.H, p.ldh) && al(p.N, p.ldn) && al(p.gamma, 0) &&
                     reinterpret_cast<uintptr_t>(p.Q) % V == 0;
    return vec ? run<E, V>(p, c) : run<E, 1>(p, c);
}

// Rows of a strided matrix: T rows of `width` bytes, `pitch` bytes apart
struct Rows {
    const void *p;
    int64_t T, width, pitch;
};
bool overlap(const Rows &a, const Rows &b)
{
    if (!a.p || !b.p || a.T == 0 || b.T == 0) return false;
    const int64_t la = (a.T - 1) * a.pitch + a.width, lb = (b.T - 1) * b.pitch + b.width;
    if (!overlaps(rng(a.p, la, 1), rng(b.p, lb, 1))) return false;
    if (a.T == 1 && b.T == 1) return true;
    // equal pitches: the columns decide
    if (a.pitch != b.pitch || a.pitch <= 0) return true;
    const int64_t diff = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
    const int64_t at = (diff % a.pitch + a.pitch) % a.pitch;   // b's column within a's row
    return at < a.width || at + b.width > a.pitch;
}

}  // namespace
}  // namespace resbm

using namespace resbm;

extern "C" resbm_status resbm_add_rmsnorm_fwd(const resbm_add_norm_desc *desc, const void *X, const void *A, const void *gamma,
                                              void *H, void *N, void *Q, float *S, void *stream)
{
    if (!desc) return RESBM_ERR_INVALID_ARG;
    const resbm_add_norm_desc &d = *desc;
    if (d.T < 0 || d.d < 1 || d.d > INT32_MAX / 4 || (d.dtype != RESBM_F32 && d.dtype != RESBM_BF16) || d.flags || !(d.eps >= 0.0f) || !(d.eps < INFINITY))
        return RESBM_ERR_INVALID_ARG;
    if (d.T > 0 && ((!N && !Q) || !Q != !S)) return RESBM_ERR_INVALID_ARG;
    if (Q && d.q_group != 0 && (d.q_group < 32 || (d.q_group & (d.q_group - 1)))) return RESBM_ERR_INVALID_ARG;
    const int64_t es = d.dtype == RESBM_BF16 ? 2 : 4, limit = INT64_MAX / 64;
    const bool t = d.T > 0;
    if (!ptr_ok(X, es, t) || !ptr_ok(A, es, false) || !ptr_ok(gamma, es, true) || !ptr_ok(H, es, false) || !ptr_ok(N, es, false) || !ptr_ok(S, 4, false))
        return RESBM_ERR_INVALID_ARG;
    // one row: its stride is never used
    auto ld = [&](int64_t v) { return d.T <= 1 ? d.d : v; };
    const int64_t ldx = ld(d.ldx), lda = ld(d.lda), ldh = ld(d.ldh), ldn = ld(d.ldn);
    auto bad = [&](const void *q, int64_t v, bool in) { return q && !(in && v == 0) && (v < d.d || !mul_ok(d.T, v) || d.T * v > limit); };
    if (bad(X, ldx, true) || bad(A, lda, true) || bad(H, ldh, false) || bad(N, ldn, false) || !mul_ok(d.T, d.d) || d.T * d.d > limit)
        return RESBM_ERR_INVALID_ARG;
    const int64_t groups = d.q_group ? (d.d + d.q_group - 1) / d.q_group : 1;
    const Rows x{X, d.T, d.d * es, ldx * es}, a{A, d.T, d.d * es, lda * es}, g{gamma, 1, d.d * es, d.d * es};
    const Rows h{H, d.T, d.d * es, ldh * es}, n{N, d.T, d.d * es, ldn * es}, q{Q, d.T, d.d, d.d}, s{S, d.T, groups * 4, groups * 4};
    const bool in_x = H && H == X && ldh == ldx, in_a = H && H == A && ldh == lda;   // in place
    if ((!in_x && overlap(h, x)) || (!in_a && overlap(h, a)) || overlap(h, g)) return RESBM_ERR_INVALID_ARG;
    for (const Rows *o : {&n, &q, &s}) {
        if (overlap(*o, x) || overlap(*o, a) || overlap(*o, g) || overlap(*o, h)) return RESBM_ERR_INVALID_ARG;
        for (const Rows *r : {&n, &q, &s})
            if (r != o && overlap(*o, *r)) return RESBM_ERR_INVALID_ARG;
    }
    Ctx c;
    resbm_status st = make_ctx(stream, &c);
    if (st != RESBM_OK || !t) return st;
    NormArgs p{X, A, gamma, H, N, static_cast<uint8_t *>(Q), S, d.T, ldx, lda, ldh, ldn, groups, (int)d.d, 0, d.eps, (float)(1.0 / (double)d.d)};
    p.group_log = d.q_group && d.q_group <= d.d ? __builtin_ctz((unsigned)d.q_group) : 30;
    const cudaError_t e = d.dtype == RESBM_F32 ? run<float>(p, c) : run<__nv_bfloat16>(p, c);
    if (e == cudaSuccess) count_launches(1);
    else cudaGetLastError();
    return finish(e);
}
