// vocab_few.cu -- the losses over the vocabulary for a handful of tokens (up to eight): the scores of single tokens. The
// head's rows are read once, by plain vector loads, and everything is done with a row while it is in registers; a tensor core's tile
// would be nearly empty, and its loads (128 bytes of a row at a time) reach half of HBM's rate.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "common.cuh"
#include "pair.cuh"
#include "tc_host.cuh"
#include "vocab.h"

namespace resbm {
namespace {

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// VEC elements (16 bytes, or one off the 16-byte grid)
template <typename E, int VEC> struct Raw {
    uint32_t w[VEC == 1 ? 1 : 4];
    __device__ __forceinline__ void load(const E *p)
    {
        if constexpr (VEC > 1) {
            const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p));
            w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
        } else if constexpr (sizeof(E) == 2) {
            w[0] = (uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16;
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        }
    }
    __device__ __forceinline__ void shared(const E *p)
    {
        if constexpr (VEC > 1) {
            const uint4 u = *reinterpret_cast<const uint4 *>(p);
            w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
        } else if constexpr (sizeof(E) == 2) {
            w[0] = (uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16;
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < (VEC == 1 ? 1 : 4); ++i) w[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (VEC == 1 || sizeof(E) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
};

// The tokens' rows in shared memory (zeros for a token without a target, whatever its row holds, and behind d)
template <typename E, int TT> __device__ __forceinline__ void stage_tokens(const FewArgs &a, E *xs)
{
    for (int i = threadIdx.x; i < TT * a.dp; i += blockDim.x) {
        const int t = i / a.dp, c = i - t * a.dp;
        const bool in = t < a.T && c < a.d && (a.label ? a.label[t] >= 0 : a.count[t] > 0);
        xs[i] = in ? static_cast<const E *>(a.X)[(int64_t)t * a.ldx + c] : from_f32<E>(0.0f);
    }
}

// The weight of word v among token t's targets
__device__ __forceinline__ float target_weight(const FewArgs &a, int t, int64_t v)
{
    if (a.label) return a.label[t] == v ? 1.0f : 0.0f;
    const int32_t *list = a.list + (int64_t)t * a.K;
    int lo = 0, hi = a.K;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    float q = 0.0f;
    for (; lo < a.K && list[lo] == v; ++lo) q += a.weight[(int64_t)t * a.K + lo];
    return q;
}

constexpr int kRows = 4;   // words at a time

// A warp takes four words at a time; lane r * TT + t then has the logit of word r and token t, and keeps the running maximum and
// sum of its token. One slot a CTA (k_join).
template <typename E, int VEC, int TT> __global__ void __launch_bounds__(256) k_few_fwd(const FewArgs a)
{
    extern __shared__ __align__(16) uint8_t few_smem[];
    E *xs = reinterpret_cast<E *>(few_smem);
    __shared__ float sm[8][TT], ss[8][TT], sz[8][TT];
    griddep_wait();
    griddep_launch_dependents();
    stage_tokens<E, TT>(a, xs);
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = lane % TT;
    const bool live = lane < kRows * TT && t < a.T;
    float most = -INFINITY, sum = 0.0f, zt = 0.0f;
    const E *W = static_cast<const E *>(a.W);
    for (int64_t v0 = ((int64_t)blockIdx.x * 8 + warp) * kRows; v0 < a.V; v0 += (int64_t)gridDim.x * 8 * kRows) {
        float acc[kRows][TT] = {};
        const E *row[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) row[r] = W + (v0 + r < a.V ? v0 + r : a.V - 1) * a.ldw;
#pragma unroll 4
        for (int c = lane * VEC; c < a.d; c += 32 * VEC) {
            Raw<E, VEC> w[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) w[r].load(row[r] + c);
#pragma unroll
            for (int k = 0; k < TT; ++k) {
                Raw<E, VEC> x;
                x.shared(xs + k * a.dp + c);
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[r][k] = fmaf(x.get(i), w[r].get(i), acc[r][k]);
            }
        }
        float z = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int k = 0; k < TT; ++k) {
#pragma unroll
                for (int o = 16; o; o >>= 1) acc[r][k] += __shfl_xor_sync(0xffffffffu, acc[r][k], o);
                if (lane == r * TT + k) z = acc[r][k];
            }
        const int64_t v = v0 + lane / TT;
        if (live && v < a.V) {
            const float q = target_weight(a, t, v);
            if (a.label) {
                if (q != 0.0f) a.zt[t] = z;
            } else if (q != 0.0f) {
                zt = fmaf(q, z, zt);
            }
            const float now = max_nan(most, z * a.c);
            if (!(now == -INFINITY)) {
                sum = fmaf(sum, exp2_approx(most - now), exp2_approx(fmaf(z, a.c, -now)));
                most = now;
            }
        }
    }
    // the lanes of a token, then the warps
#pragma unroll
    for (int o = TT; o < kRows * TT; o <<= 1) {
        const float m = __shfl_xor_sync(0xffffffffu, most, o), s = __shfl_xor_sync(0xffffffffu, sum, o);
        zt += __shfl_xor_sync(0xffffffffu, zt, o);
        const float now = max_nan(most, m);
        if (!(now == -INFINITY)) sum = sum * exp2_approx(most - now) + s * exp2_approx(m - now);
        most = now;
    }
    if (lane < TT) {
        sm[warp][lane] = most;
        ss[warp][lane] = sum;
        sz[warp][lane] = zt;
    }
    __syncthreads();
    const int k = threadIdx.x;
    if (k < TT && k < a.T) {
        most = sm[0][k];
        sum = ss[0][k];
        zt = sz[0][k];
        for (int w = 1; w < 8; ++w) {
            const float now = max_nan(most, sm[w][k]);
            if (!(now == -INFINITY)) sum = sum * exp2_approx(most - now) + ss[w][k] * exp2_approx(sm[w][k] - now);
            most = now;
            zt += sz[w][k];
        }
        a.stat[(int64_t)blockIdx.x * a.tp + k] = make_float2(most, sum);
        if (!a.label) a.zt[(int64_t)blockIdx.x * a.tp + k] = zt;
    }
}

// A CTA takes four words at a time, each thread NV vectors of their rows: the logits by a sum over the CTA, their dz, then
// the rows' of dW, and dX's sums in registers. W is read once, dW written once, and dX leaves as a slot a CTA.
template <typename E, int VEC, int NV, int TT> __global__ void __launch_bounds__(256) k_few_bwd(const FewArgs a)
{
    extern __shared__ __align__(16) uint8_t few_smem[];
    E *xs = reinterpret_cast<E *>(few_smem);
    __shared__ float part[2][8][kRows * TT], dzs[2][kRows * TT];
    griddep_wait();
    griddep_launch_dependents();
    stage_tokens<E, TT>(a, xs);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // thread r * TT + t makes dz of word r and token t
    const int my = threadIdx.x < kRows * TT ? (int)threadIdx.x % TT : 0;
    const bool live = threadIdx.x < kRows * TT && my < a.T && (a.label ? a.label[my] >= 0 : a.count[my] > 0);
    float lse2 = 0.0f, grad = 0.0f;
    if (live) {
        lse2 = a.lse[my] * 1.4426950408889634f;
        grad = a.dloss[(int64_t)my * a.dloss_step] * a.tau;
        if (a.label ? a.label[my] >= a.V : a.bad[my] != 0.0f) grad = NAN;
    }
    __syncthreads();
    float dx[TT][NV * VEC] = {};
    const E *W = static_cast<const E *>(a.W);
    E *dW = static_cast<E *>(a.dW);
    Raw<E, VEC> w[kRows][NV];
    auto load = [&](int64_t v0) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int c = (n * 256 + (int)threadIdx.x) * VEC;
                if (c < a.d && v0 + r < a.V) w[r][n].load(W + (v0 + r) * a.ldw + c);
                else w[r][n].zero();
            }
    };
    int side = 0;
    for (int64_t v0 = (int64_t)blockIdx.x * kRows; v0 < a.V; v0 += (int64_t)gridDim.x * kRows, side ^= 1) {
        load(v0);
        float acc[kRows][TT] = {};
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * 256 + (int)threadIdx.x) * VEC;
            if (c < a.d) {
#pragma unroll
                for (int k = 0; k < TT; ++k) {
                    Raw<E, VEC> x;
                    x.shared(xs + k * a.dp + c);
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
#pragma unroll
                        for (int i = 0; i < VEC; ++i) acc[r][k] = fmaf(x.get(i), w[r][n].get(i), acc[r][k]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int k = 0; k < TT; ++k) {
#pragma unroll
                for (int o = 16; o; o >>= 1) acc[r][k] += __shfl_xor_sync(0xffffffffu, acc[r][k], o);
                if (lane == 0) part[side][warp][r * TT + k] = acc[r][k];
            }
        __syncthreads();
        if (threadIdx.x < kRows * TT) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) z += part[side][i][threadIdx.x];
            const int64_t v = v0 + threadIdx.x / TT;
            dzs[side][threadIdx.x] = live && v < a.V ? (exp2_approx(fmaf(z, a.c, -lse2)) - target_weight(a, my, v)) * grad : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * 256 + (int)threadIdx.x) * VEC;
            if (c >= a.d) continue;
            if (a.dX) {
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int k = 0; k < TT; ++k) {
                        const float g = dzs[side][r * TT + k];
#pragma unroll
                        for (int i = 0; i < VEC; ++i) dx[k][n * VEC + i] = fmaf(g, w[r][n].get(i), dx[k][n * VEC + i]);
                    }
            }
            if (dW) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (v0 + r >= a.V) break;
                    float y[VEC] = {};
#pragma unroll
                    for (int k = 0; k < TT; ++k) {
                        Raw<E, VEC> x;
                        x.shared(xs + k * a.dp + c);
                        const float g = dzs[side][r * TT + k];
#pragma unroll
                        for (int i = 0; i < VEC; ++i) y[i] = fmaf(g, x.get(i), y[i]);
                    }
                    E *dst = dW + (v0 + r) * a.d + c;
                    if constexpr (VEC == 1) {
                        *dst = from_f32<E>(y[0]);
                    } else if constexpr (sizeof(E) == 4) {
                        __stcs(reinterpret_cast<float4 *>(dst), make_float4(y[0], y[1], y[2], y[3]));
                    } else {
                        uint32_t o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
                            o[i] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        __stcs(reinterpret_cast<uint4 *>(dst), make_uint4(o[0], o[1], o[2], o[3]));
                    }
                }
            }
        }
    }
    if (!a.dX) return;
#pragma unroll
    for (int k = 0; k < TT; ++k) {
        if (k >= a.T) break;
        float *dst = a.slots + ((int64_t)blockIdx.x * a.T + k) * a.dp;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int c = (n * 256 + (int)threadIdx.x) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i < a.d) dst[c + i] = dx[k][n * VEC + i];
        }
    }
}

// dX of a token: the CTAs' sums in order. 32 columns a CTA, eight threads each over the slots.
template <typename E> __global__ void __launch_bounds__(256) k_few_finish(const FewArgs a, int slots)
{
    __shared__ float sh[8][32];
    griddep_wait();
    griddep_launch_dependents();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x, t = blockIdx.y;
    float sum = 0.0f;
    if (c < a.d) {
#pragma unroll 8
        for (int s = y; s < slots; s += 8) sum += a.slots[((int64_t)s * a.T + t) * a.dp + c];
    }
    sh[y][x] = sum;
    __syncthreads();
    if (y == 0 && c < a.d) {
        for (int i = 1; i < 8; ++i) sum += sh[i][x];
        static_cast<E *>(a.dX)[(int64_t)t * a.d + c] = from_f32<E>(sum);
    }
}

template <typename K> cudaError_t go(K kernel, int smem, int grid, const FewArgs &a, const Ctx &c, std::atomic<uint8_t> (&done)[kMaxDev])
{
    cudaError_t e = smem > 40 * 1024 ? ensure_smem(kernel, 64 * 1024, c.device, done) : cudaSuccess;
    return e != cudaSuccess ? e : launch(kernel, dim3((unsigned)grid), dim3(256), (size_t)smem, c.stream, a);
}

template <typename E, int VEC, int TT> cudaError_t fwd(const FewArgs &a, int grid, const Ctx &c)
{
    static std::atomic<uint8_t> done[kMaxDev];
    return go(k_few_fwd<E, VEC, TT>, TT * a.dp * (int)sizeof(E), grid, a, c, done);
}
template <typename E, int VEC, int NV, int TT> cudaError_t bwd(const FewArgs &a, int grid, const Ctx &c)
{
    static std::atomic<uint8_t> done[kMaxDev];
    return go(k_few_bwd<E, VEC, NV, TT>, TT * a.dp * (int)sizeof(E), grid, a, c, done);
}

int tokens_of(int64_t T) { return T <= 1 ? 1 : T <= 4 ? 4 : 8; }

template <typename E> cudaError_t run(const FewArgs &a, const Ctx &c, int *launches)
{
    constexpr int V16 = 16 / (int)sizeof(E);
    const bool vec = a.d % V16 == 0 && al16(a.W) && (a.V == 1 || a.ldw % V16 == 0) && (!a.bwd || !a.dW || al16(a.dW));
    const int tt = tokens_of(a.T);
    *launches = 1;
    if (!a.bwd) {
        const int grid = few_slots(a.V, false, c.sm_count);
        if (vec) return tt == 1 ? fwd<E, V16, 1>(a, grid, c) : tt == 4 ? fwd<E, V16, 4>(a, grid, c) : fwd<E, V16, 8>(a, grid, c);
        return tt == 1 ? fwd<E, 1, 1>(a, grid, c) : tt == 4 ? fwd<E, 1, 4>(a, grid, c) : fwd<E, 1, 8>(a, grid, c);
    }
    const int grid = few_slots(a.V, true, c.sm_count);
    cudaError_t e;
    constexpr int N1 = sizeof(E) == 2 ? 1 : 2;   // vectors of a row of up to 2048
    if (tt == 8) e = vec ? bwd<E, V16, N1, 8>(a, grid, c) : bwd<E, 1, 8, 8>(a, grid, c);
    else if (a.d <= 2048) {
        if (vec) e = tt == 1 ? bwd<E, V16, N1, 1>(a, grid, c) : bwd<E, V16, N1, 4>(a, grid, c);
        else e = tt == 1 ? bwd<E, 1, 8, 1>(a, grid, c) : bwd<E, 1, 8, 4>(a, grid, c);
    } else {
        if (vec) e = tt == 1 ? bwd<E, V16, 2 * N1, 1>(a, grid, c) : bwd<E, V16, 2 * N1, 4>(a, grid, c);
        else e = tt == 1 ? bwd<E, 1, 16, 1>(a, grid, c) : bwd<E, 1, 16, 4>(a, grid, c);
    }
    if (e == cudaSuccess && a.dX) {
        e = launch(k_few_finish<E>, dim3((unsigned)((a.d + 31) / 32), (unsigned)a.T), dim3(256), 0, c.stream, a, grid);
        ++*launches;
    }
    return e;
}

}  // namespace

bool few_tokens(int64_t T, int64_t d, int64_t es, bool bwd)
{
    if (T < 1 || T > kFewTokens) return false;
    const int tt = tokens_of(T);
    if (tt * ((d + 7) / 8 * 8) * es > 64 * 1024) return false;
    return !bwd || d <= (tt == 8 ? 2048 : 4096);
}

int few_slots(int64_t V, bool bwd, int sms)
{
    const int64_t per = bwd ? kRows : 8 * kRows;
    return (int)std::max<int64_t>(1, std::min<int64_t>((V + per - 1) / per, std::min(kFewSlots, 2 * sms)));
}

cudaError_t few_run(const FewArgs &a, bool f32, const Ctx &c, int *launches) { return f32 ? run<float>(a, c, launches) : run<__nv_bfloat16>(a, c, launches); }

}  // namespace resbm
