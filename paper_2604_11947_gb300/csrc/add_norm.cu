// add_norm.cu -- resbm_add_rmsnorm_fwd: h = x + a, n = h / sqrt(mean h^2 + eps) * gamma, n in the activations'
// type and / or in e4m3 with scales (include/resbm_train.h).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

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
    float eps;
    float inv_d;
    float part, whole;            // 1 / d as two factors, a square's and a sum's: a power of two of at most 1 / d, and the rest
};

template <int V> __device__ __forceinline__ void scale_by(float (&f)[V], float c)
{
#pragma unroll
    for (int i = 0; i < V; i += 2) split(pair(f[i], f[i + 1]) * both(c), f[i], f[i + 1]);
}

// 16 bytes of a row: 8 bf16 or 4 fp32 elements
template <typename E> struct Vec {
    static constexpr int V = 16 / (int)sizeof(E);
    uint32_t w[4];

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
    // the sum of the squares, each times c
    __device__ __forceinline__ float squares(float c) const
    {
        Pair s = both(0.0f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) s = fma(get(i) * both(c), get(i), s);
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
    // the first n elements stay, the others become zero
    __device__ __forceinline__ void keep(int n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) w[i] = n >= 2 * i + 2 ? w[i] : n == 2 * i + 1 ? w[i] & 0xFFFFu : 0u;
            else w[i] = n > i ? w[i] : 0u;
        }
    }
};
// The e4m3 codes of a vector
template <int V> struct Codes {
    uint32_t w[V / 4];
    __device__ __forceinline__ explicit Codes(const float (&f)[V])
    {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = e4m3x4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
    }
    __device__ __forceinline__ void store(uint8_t *p) const
    {
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(p) = w[0];
    }
};

// Bytes 4 WORDS + bits / 8 .. of lo followed by hi, 4 NW of them (BYTES: bits need not be 0)
template <int NW, int WORDS, bool BYTES> __device__ __forceinline__ void realign(const uint32_t (&lo)[NW], const uint32_t (&hi)[NW], int bits, uint32_t (&out)[NW])
{
    uint32_t x[2 * NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        x[i] = lo[i];
        x[NW + i] = hi[i];
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) out[i] = BYTES ? __funnelshift_r(x[i + WORDS], x[i + WORDS + 1], bits) : x[i + WORDS];
}

// f with `words` (0 .. NW - 1, the same in the whole warp) as a constant
template <int NW, typename F> __device__ __forceinline__ void with_words(int words, F f)
{
    if constexpr (NW == 1) {
        f(std::integral_constant<int, 0>());
    } else if constexpr (NW == 2) {
        if (words) f(std::integral_constant<int, 1>());
        else f(std::integral_constant<int, 0>());
    } else {
        switch (words) {
        case 0: f(std::integral_constant<int, 0>()); break;
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        default: f(std::integral_constant<int, 3>()); break;
        }
    }
}

// A row whose first element is anywhere: element j of the row is byte `off` + j * size of the words from `base`
template <typename E> struct Shifted {
    const char *base;
    int off;
    __device__ __forceinline__ explicit Shifted(const E *row, int word)
    {
        off = (int)(reinterpret_cast<uintptr_t>(row) & (uintptr_t)(word - 1));
        base = reinterpret_cast<const char *>(row) - off;
    }
};

// Vectors q, q + 32, ... of a row of d elements that starts anywhere: each from the two 16-byte words that hold it, no word
// without an element of the row (past its end the last one again); elements past the row are zero.
template <typename E, int KV> __device__ __forceinline__ void load_shifted(Vec<E> (&r)[KV], const E *from, int q, int d)
{
    constexpr int V = Vec<E>::V;
    const Shifted<E> row(from, 16);
    const int end = (row.off + d * (int)sizeof(E) - 1) >> 4;   // the last word
    auto word = [&](Vec<E> &v, int i) { v.load(reinterpret_cast<const E *>(row.base + (int64_t)16 * min(i, end))); };
    if (row.off) {
        with_words<4>(row.off >> 2, [&](auto words) {
            Vec<E> lo[KV], hi[KV];
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                word(lo[k], q + 32 * k);
                word(hi[k], q + 32 * k + 1);
            }
#pragma unroll
            for (int k = 0; k < KV; ++k) realign<4, decltype(words)::value, sizeof(E) != 4>(lo[k].w, hi[k].w, 8 * (row.off & 3), r[k].w);
        });
    } else {
#pragma unroll
        for (int k = 0; k < KV; ++k) word(r[k], q + 32 * k);
    }
#pragma unroll
    for (int k = 0; k < KV; ++k)
        if (V * (q + 32 * k + 1) > d) r[k].keep(d - V * (q + 32 * k));
}

// Element `lane` of the words that lane `from` holds
template <typename T, int NW> __device__ __forceinline__ T element(const uint32_t (&w)[NW], int from, int lane)
{
    constexpr int kSize = sizeof(T);
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const uint32_t x = __shfl_sync(0xffffffffu, w[i], from);
        r = lane * kSize / 4 == i ? x : r;
    }
    return (T)(kSize == 4 ? r : r >> (8 * (lane * kSize % 4)));
}

// A warp's KV vectors, neighbours in lanes and then in k, from vector q0 (lane 0, k = 0) on, into a row that starts at any
// element (T: what an element is stored as, NW words a vector): whole words where the warp has all of one; the elements
// before its first whole word and behind its last, fewer than a word's each, one a lane. get(k, out): the words of vector k.
template <typename T, int NW, int KV, typename Get> __device__ __forceinline__ void store_shifted(T *row, int q0, int lane, int d, Get get)
{
    constexpr int kSize = sizeof(T), V = 4 * NW / kSize, kWord = 4 * NW;
    const Shifted<T> at(row, kWord);
    const int o = at.off / kSize;                                   // elements before the row in its first word
    const int first = q0 * V, last = min(first + 32 * KV * V, d);   // the warp's elements
    uint32_t tail[NW] = {};                                         // the last, partial word
    int behind = -1;                                                // its first element
    // `out`: the word that ends in vector k, from element `from` on
    auto put = [&](const uint32_t (&out)[NW], int from) {
        if (from >= first && from + V <= last) {
            char *const p = const_cast<char *>(at.base) + (int64_t)(from + o) * kSize;
            if constexpr (NW == 4) *reinterpret_cast<uint4 *>(p) = make_uint4(out[0], out[1], out[2], out[3]);
            else if constexpr (NW == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(out[0], out[1]);
            else *reinterpret_cast<uint32_t *>(p) = out[0];
        } else if (from >= first && from < last) {
            behind = from;
#pragma unroll
            for (int i = 0; i < NW; ++i) tail[i] = out[i];
        }
    };
    const int start = (q0 + lane) * V - o;
    if (o) {
        const int n = kWord - at.off, bits = 8 * (n & 3);
        with_words<NW>(n >> 2, [&](auto words) {
            constexpr int kWords = decltype(words)::value;
            uint32_t before[NW] = {};                               // lane 31's words of the previous k, in lane 0
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                uint32_t own[NW], prev[NW], out[NW];
                get(k, own);
                if (k == 0) {
                    const T x = element<T, NW>(own, 0, lane);
                    if (lane < V - o && first + lane < last) row[first + lane] = x;
                }
#pragma unroll
                for (int i = 0; i < NW; ++i) {
                    const uint32_t left = __shfl_sync(0xffffffffu, own[i], (lane + 31) & 31);
                    prev[i] = lane == 0 ? before[i] : left;
                    before[i] = left;
                }
                realign<NW, kWords, kSize != 4>(prev, own, bits, out);
                const int from = start + 32 * k * V;
                put(out, from);
                if (k == KV - 1 && lane == 31 && from + V < last) {   // the word that only begins in the last vector
                    const uint32_t none[NW] = {};
                    behind = from + V;
                    realign<NW, kWords, kSize != 4>(own, none, bits, tail);
                }
            }
        });
    } else {
#pragma unroll
        for (int k = 0; k < KV; ++k) {
            uint32_t own[NW];
            get(k, own);
            put(own, start + 32 * k * V);
        }
    }
    const unsigned has = __ballot_sync(0xffffffffu, behind >= 0);   // (one lane at most)
    if (has) {
        const int src = __ffs(has) - 1, from = __shfl_sync(0xffffffffu, behind, src);
        const T x = element<T, NW>(tail, src, lane);
        if (lane < V && from + lane < last) row[from + lane] = x;
    }
}

// CTAs (of the most threads) that an SM holds at least, which bounds the registers. A CTA a row: 64 registers a thread;
// with three vectors and no bound the compiler takes 77 (bf16 T = 65536, d = 4096 to e4m3 305 us instead of 265, the
// realigned T = 10000, d = 5001 162 instead of 102). A warp a row: 64, but 80 for four bf16 vectors, whose realignment
// needs them (T = 20000, d = 1001 57 us without a bound, 38 at 80, 41 at 64; two vectors, d = 301: 78 without, 70 at 64).
// Eight vectors a thread need all that they can get.
template <typename E, int KV, int MAXT> constexpr int min_ctas()
{
    return MAXT == 32 ? (KV == 4 && sizeof(E) == 2 ? 3 : 4) : KV <= 4 ? 2 : 1;
}

// The row in registers: a warp a row (MAXT = 32, in CTAs of eight) or a CTA of up to MAXT threads a row, each thread with
// KV vectors of 16 bytes, a warp's vectors one contiguous piece of the row. X and A are read once, H, N, Q and S written
// once. The sum of squares goes through a fixed shuffle tree and the warps' sums through another. SHIFT: rows that start
// or end off the vectors' alignment; every tensor's row is then realigned by itself on its way in and out (T = 20000,
// d = 1001, bf16: 34 us; single elements took 90 instructions each and 67 us, the shift of words by selects 38).
template <typename E, int KV, int MAXT, bool SHIFT>
__global__ void __launch_bounds__(MAXT == 32 ? 256 : MAXT, min_ctas<E, KV, MAXT>()) k_add_norm(const __grid_constant__ NormArgs p)
{
    using L = Vec<E>;
    constexpr int V = L::V, kLogV = V == 8 ? 3 : 2;
    constexpr bool kWide = MAXT > 32;                // a CTA a row
    constexpr int kRows = kWide ? 1 : 8;
    using Bits = typename std::conditional<sizeof(E) == 2, uint16_t, uint32_t>::type;
    __shared__ float sums[32];
    __shared__ uint32_t most[KV * 32];               // the largest |n| of every 32 vectors, or of a warp's
    __shared__ float factor[KV * 32];                // 448 over a group's
    const int lane = threadIdx.x & 31, warp = kWide ? (int)threadIdx.x >> 5 : 0, warps = kWide ? (int)blockDim.x >> 5 : 1;
    const int nv = (p.d + V - 1) / V, q0 = warp * 32 * KV, qt = q0 + lane;   // qt + 32 k: this thread's vectors
    const E *const gamma = static_cast<const E *>(p.gamma);
    griddep_wait();
    griddep_launch_dependents();
    auto load = [&](L (&r)[KV], const E *row) {
        if constexpr (SHIFT) {
            load_shifted<E, KV>(r, row, qt, p.d);
        } else {
            const E *const at = row + qt * V;
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                if (qt + 32 * k < nv) r[k].load(at + 32 * k * V);
                else r[k].zero();
            }
        }
    };
    // r(k): vector k as an L
    auto store = [&](E *row, auto r) {
        if constexpr (SHIFT) {
            store_shifted<Bits, 4, KV>(reinterpret_cast<Bits *>(row), q0, lane, p.d, [&](int k, uint32_t (&w)[4]) {
                const L x = r(k);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = x.w[i];
            });
        } else {
            E *const at = row + qt * V;
#pragma unroll
            for (int k = 0; k < KV; ++k)
                if (qt + 32 * k < nv) r(k).store(at + 32 * k * V);
        }
    };
    for (int64_t t = (int64_t)blockIdx.x * kRows + (kWide ? 0 : threadIdx.x >> 5); t < p.T; t += (int64_t)gridDim.x * kRows) {
        L h[KV], b[KV];
        load(h, static_cast<const E *>(p.X) + t * p.ldx);
        if (p.A) {
            load(b, static_cast<const E *>(p.A) + t * p.lda);
#pragma unroll
            for (int k = 0; k < KV; ++k) h[k].add(b[k]);
        }
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < KV; ++k) s += h[k].squares(p.part);   // (of h as stored)
        if (p.H) {
            // (in place: a word of X or A that two threads read is read by both before either stores)
            if (SHIFT && kWide) __syncthreads();
            else if (SHIFT) __syncwarp();
            store(static_cast<E *>(p.H) + t * p.ldh, [&](int k) { return h[k]; });
        }
        s *= p.whole;   // (a thread's share of the mean. A square, a thread's sum and the row's own could leave fp32's range where
                        // the mean does not; scaled by a power of two before the square, none does, and no bit changes)
        load(b, gamma);   // on its way while the sums travel
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (kWide) {
            if (lane == 0) sums[warp] = s;
            __syncthreads();
            s = lane < warps ? sums[lane] : 0.0f;
#pragma unroll
            for (int o = MAXT >= 1024 ? 16 : MAXT / 64; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (MAXT < 1024) s = __shfl_sync(0xffffffffu, s, 0);
        }
        const float rstd = 1.0f / sqrtf(s + p.eps);
        float n[KV][V];
#pragma unroll
        for (int k = 0; k < KV; ++k) h[k].scaled(rstd, b[k], n[k]);
        if (p.N)
            store(static_cast<E *>(p.N) + t * p.ldn, [&](int k) {
                L r;
                r.put(n[k]);
                return r;
            });
        if (p.Q) {
            // the largest |n| of a group: over the lanes that share it; over a warp's pieces of 32 vectors, in shared
            // memory where other warps have some of them; or, for the whole row, over the warps
            const int lanes_log = p.group_log - kLogV;
            uint32_t am[KV];
#pragma unroll
            for (int k = 0; k < KV; ++k) {
                float m = fabsf(n[k][0]);
#pragma unroll
                for (int i = 1; i < V; ++i) m = max_nan(m, fabsf(n[k][i]));
                am[k] = abs_bits(m);
            }
            float *const S = p.S + t * p.groups;
            bool mine = true;   // whether this thread writes its groups' scales
            if (p.groups == 1) {
                uint32_t m = am[0];
#pragma unroll
                for (int k = 1; k < KV; ++k) m = max(m, am[k]);
                m = __reduce_max_sync(0xffffffffu, m);
                if (kWide) {
                    if (lane == 0) most[warp] = m;
                    __syncthreads();
                    m = __reduce_max_sync(0xffffffffu, lane < warps ? most[lane] : 0u);
                }
                const E4m3Scale c = e4m3_scale(m);
#pragma unroll
                for (int k = 0; k < KV; ++k) scale_by(n[k], c.inv);
                if (qt == 0) S[0] = c.scale;
                mine = false;
            } else if (lanes_log < 5) {
                for (int o = 1 << lanes_log >> 1; o > 0; o >>= 1)
#pragma unroll
                    for (int k = 0; k < KV; ++k) am[k] = max(am[k], __shfl_xor_sync(0xffffffffu, am[k], o));
            } else {
                const int pieces_log = lanes_log - 5;
#pragma unroll
                for (int k = 0; k < KV; ++k) am[k] = __reduce_max_sync(0xffffffffu, am[k]);
                if (pieces_log > 0 && kWide) {   // a warp a group, from shared memory
                    if (lane == 0)
#pragma unroll
                        for (int k = 0; k < KV; ++k) most[warp * KV + k] = am[k];
                    __syncthreads();
                    for (int g = warp; g < (int)p.groups; g += warps) {
                        uint32_t m = 0;
                        for (int c = lane; c < 1 << pieces_log; c += 32)
                            if ((g << pieces_log) + c < warps * KV) m = max(m, most[(g << pieces_log) + c]);
                        const E4m3Scale c = e4m3_scale(__reduce_max_sync(0xffffffffu, m));
                        if (lane == 0) {
                            factor[g] = c.inv;
                            S[g] = c.scale;
                        }
                    }
                    __syncthreads();
#pragma unroll
                    for (int k = 0; k < KV; ++k)
                        if (qt + 32 * k < nv) scale_by(n[k], factor[(warp * KV + k) >> pieces_log]);
                    mine = false;
                } else if (pieces_log > 0) {
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
            if (mine) {
#pragma unroll
                for (int k = 0; k < KV; ++k) {
                    const E4m3Scale c = e4m3_scale(am[k]);
                    scale_by(n[k], c.inv);
                    const int q = qt + 32 * k;
                    if (q < nv && (q & ((1 << lanes_log) - 1)) == 0) S[q >> lanes_log] = c.scale;
                }
            }
            uint8_t *const Q = p.Q + t * p.d;
            if constexpr (SHIFT) {
                store_shifted<uint8_t, V / 4, KV>(Q, q0, lane, p.d, [&](int k, uint32_t (&w)[V / 4]) {
                    const Codes<V> c(n[k]);
#pragma unroll
                    for (int i = 0; i < V / 4; ++i) w[i] = c.w[i];
                });
            } else {
#pragma unroll
                for (int k = 0; k < KV; ++k)
                    if (qt + 32 * k < nv) Codes<V>(n[k]).store(Q + (qt + 32 * k) * V);
            }
        }
        if (kWide) __syncthreads();   // sums, most and factor are this row's until here
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

template <typename E, int KV, int MAXT> cudaError_t launch(const NormArgs &p, bool shift, const Ctx &c)
{
    const int64_t rows = MAXT > 32 ? 1 : 8, nv = (p.d + Vec<E>::V - 1) / Vec<E>::V;
    const unsigned grid = (unsigned)std::min<int64_t>((p.T + rows - 1) / rows, INT32_MAX);
    const unsigned threads = MAXT > 32 ? (unsigned)((nv + KV * 32 - 1) / (KV * 32)) * 32 : 256;
    return launch_pdl(shift ? k_add_norm<E, KV, MAXT, true> : k_add_norm<E, KV, MAXT, false>, dim3(grid), dim3(threads), 0, c, p);
}

template <typename E> cudaError_t run(const NormArgs &p, const Ctx &c)
{
    // whole vectors where every row of every tensor starts and ends at a multiple of 16 bytes (Q: of a vector's codes)
    constexpr int V = Vec<E>::V;
    auto al = [](const void *q, int64_t ld) { return !q || (reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % V == 0); };
    const bool shift = !(p.d % V == 0 && al(p.X, p.ldx) && al(p.A, p.lda) && al(p.H, p.ldh) && al(p.N, p.ldn) && al(p.gamma, 0) &&
                         reinterpret_cast<uintptr_t>(p.Q) % V == 0);
    const int64_t nv = (p.d + V - 1) / V;
    // A warp a row up to 128 vectors (no barrier), then CTAs of three vectors a thread: against two and four at bf16
    // d = 4096 to e4m3 266 us (274, 306), d = 8192 138 (160, 192), d = 2048 41.3 (41.3, 43.2). Widths that are always
    // realigned take four, since the words at a warp's ends cost as much again: d = 2001 57 us (three 63, two 67, six 95),
    // fp32 d = 1001 50 (58, 62, 71). The width alone decides, so that the sums' order does not depend on addresses.
    if (nv <= 32) return launch<E, 1, 32>(p, shift, c);
    if (nv <= 64) return launch<E, 2, 32>(p, shift, c);
    if (nv <= 96) return launch<E, 3, 32>(p, shift, c);
    if (nv <= 128) return launch<E, 4, 32>(p, shift, c);
    if (nv <= 512 * 3 && p.d % V == 0) return launch<E, 3, 512>(p, shift, c);
    if (nv <= 512 * 4) return launch<E, 4, 512>(p, shift, c);
    if (nv <= 512 * 8) return launch<E, 8, 512>(p, shift, c);
    const unsigned grid = (unsigned)std::min<int64_t>(p.T, (int64_t)c.sm_count * 2);
    return launch_pdl(k_add_norm_long<E>, dim3(grid), dim3(1024), 0, c, p);
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
    int log;
    const double m = frexp(1.0 / (double)d.d, &log);   // 1 / d = m 2^log with m from 0.5 to under 1
    p.part = (float)ldexp(1.0, log - 1);
    p.whole = (float)(2.0 * m);
    p.group_log = d.q_group && d.q_group <= d.d ? __builtin_ctz((unsigned)d.q_group) : 30;
    const cudaError_t e = d.dtype == RESBM_F32 ? run<float>(p, c) : run<__nv_bfloat16>(p, c);
    if (e == cudaSuccess) count_launches(1);
    else cudaGetLastError();
    return finish(e);
}
