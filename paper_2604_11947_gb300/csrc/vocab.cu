// vocab.cu -- the losses over the vocabulary (include/resbm_vocab.h): the small kernels around the products of
// vocab_gemm.cuh, the plan of a call, and the C entry points.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "abi.h"
#include "resbm_vocab.h"
#include "tc_common.cuh"
#include "tc_host.cuh"
#include "vocab.h"
#include "vocab_gemm.cuh"

namespace resbm {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---- the targets of a distillation ---------------------------------------------------------------
// A warp a token: q = softmax of its entries' teacher logits over tau (the largest taken off first: the lowest value of the type, over a tau
// under 1, is no number), sum q log q, and the entries in ascending order of
// their words (the products' tiles look theirs up by bisection), ranked by counting: K^2 / 32 comparisons a lane, 128 at K = 64.
template <typename E>
__global__ void __launch_bounds__(256) k_targets(const int64_t *__restrict__ index, const E *__restrict__ teacher, int64_t T, int K, int64_t V,
                                                 float tau, int2 *__restrict__ list, float *__restrict__ ent, float *__restrict__ bad, int32_t *__restrict__ count)
{
    extern __shared__ int32_t sh_key[];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    int32_t *key = sh_key + (threadIdx.x >> 5) * K;
    for (int64_t t = blockIdx.x * (int64_t)warps + (threadIdx.x >> 5); t < T; t += (int64_t)gridDim.x * warps) {
        const int64_t *ix = index + t * K;
        const E *tl = teacher + t * K;
        float most = -INFINITY;
        int have = 0, wrong = 0;
        for (int k = lane; k < K; k += 32) {
            const int64_t i = ix[k];
            key[k] = i < 0 || i >= V ? INT32_MAX : (int32_t)i;
            if (i < 0) continue;
            ++have;
            wrong |= i >= V;
            most = max_nan(most, to_f32(tl[k]));
        }
        float sum = 0.0f;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
            have += __shfl_xor_sync(0xffffffffu, have, o);
            wrong |= __shfl_xor_sync(0xffffffffu, wrong, o);
        }
        for (int k = lane; k < K; k += 32)
            if (ix[k] >= 0) sum += expf((to_f32(tl[k]) - most) / tau);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float inv = 1.0f / sum, log_sum = logf(sum);
        __syncwarp();   // (key)
        float h = 0.0f;
        for (int k = lane; k < K; k += 32) {
            const int32_t mine = key[k];
            int rank = 0;
            for (int j = 0; j < K; ++j) rank += key[j] < mine || (key[j] == mine && j < k);
            float q = 0.0f;
            if (ix[k] >= 0) {
                const float x = (to_f32(tl[k]) - most) / tau;
                q = expf(x) * inv;
                if (!(q == 0.0f)) h = fmaf(q, x - log_sum, h);
            }
            list[t * K + rank] = make_int2(mine, __float_as_int(q));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) h += __shfl_xor_sync(0xffffffffu, h, o);
        if (lane == 0) {
            ent[t] = wrong ? NAN : h;
            bad[t] = wrong ? NAN : 0.0f;
            count[t] = have;
        }
        __syncwarp();
    }
}

// ---- the tokens in use -----------------------------------------------------------------------------
// The common factor of the losses' gradients, taken out of dz before its rounding to bf16: the dz of a token's label is next to -dloss
// as long as the model knows nothing of it, and where dloss is one number for all (the mean over n tokens: 1 / n) its rounding is
// the same for all, an error of dX and dW of up to 2^-8 that no sum averages (T = 24, V = 24141, d = 2480: 2.5e-3 off, without it
// 1.9e-3; the outputs' rounding alone is 1.7e-3).
struct LossScale {
    const float *dloss;   // null: none is asked for
    int each;
    float tau;
    float *out;           // the factor, and that times tau
    // bits of a value that can be the factor, in ascending order: 0 for infinities and NaN
    __device__ __forceinline__ uint32_t bits(int64_t t) const
    {
        const uint32_t b = __float_as_uint(dloss[t]) & 0x7FFFFFFFu;
        return b < 0x7F800000u ? b : 0u;
    }
    // n tokens in use, of which `top` is the largest; where there are none a dloss of infinity (1 / 0) gives zeros
    __device__ __forceinline__ void put(int n, uint32_t top) const
    {
        const float s = n == 0 ? 1.0f : !each ? dloss[0] : top ? __uint_as_float(top) : 1.0f;
        out[0] = s;
        out[1] = s * tau;
    }
};

// token[r] = the r-th token with a target, row[t] = its r or -1, *n = how many. One cluster of eight CTAs, a contiguous run of the
// tokens a warp, counted and then written. (One CTA with eight loads a thread, one after the other: 27 us at T = 16384; this 5.)
constexpr int kScanCtas = 8;
__global__ void __cluster_dims__(kScanCtas) __launch_bounds__(1024) k_scan(const int64_t *__restrict__ label, const int32_t *__restrict__ count, int T,
                                                                           int32_t *__restrict__ n, int32_t *__restrict__ token, int32_t *__restrict__ row,
                                                                           const LossScale scale)
{
    __shared__ int sums[32], total;
    __shared__ uint32_t tops[32], top_all;
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = (int)cluster_rank();
    const int per = ((T + kScanCtas * 32 - 1) / (kScanCtas * 32) + 31) / 32 * 32;
    const int64_t first = ((int64_t)rank * 32 + warp) * per;
    const int p0 = (int)(first < T ? first : T), p1 = (int)(first + per < T ? first + per : T);
    auto has = [&](int t) { return t < p1 && (label ? label[t] >= 0 : count[t] > 0); };
    int mine = 0;
    uint32_t top = 0;
    const bool tops_too = scale.dloss && scale.each;
#pragma unroll 4
    for (int p = p0; p < p1; p += 32) {
        const bool h = has(p + lane);
        mine += __popc(__ballot_sync(0xffffffffu, h));
        if (tops_too && h) top = max(top, scale.bits(p + lane));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) {
        sums[warp] = mine;
        tops[warp] = top;
    }
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
        before += w < warp ? sums[w] : 0;
        all += sums[w];
        top = max(top, tops[w]);
    }
    if (threadIdx.x == 0) {
        total = all;
        top_all = top;
    }
    cluster_sync();
    int whole = 0;
    for (int c = 0; c < kScanCtas; ++c) {
        int v;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(map_shared(smem_addr(&total), (uint32_t)c)));
        if (c < rank) before += v;
        whole += v;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_shared(smem_addr(&top_all), (uint32_t)c)));
        top = max(top, (uint32_t)v);
    }
    for (int p = p0; p < p1; p += 32) {
        const bool h = has(p + lane);
        const uint32_t who = __ballot_sync(0xffffffffu, h);
        const int at = before + __popc(who & ((1u << lane) - 1));
        if (p + lane < p1) row[p + lane] = h ? at : -1;
        if (h) token[at] = p + lane;
        before += __popc(who);
    }
    if (rank == 0 && threadIdx.x == 0) {
        *n = whole;
        if (scale.dloss) scale.put(whole, top);
    }
    cluster_sync();   // no CTA leaves while another reads its total
}

// ---- operands with 16-byte rows --------------------------------------------------------------------
// One row of them, by a warp
template <typename E, int SPLIT>
__device__ __forceinline__ void pack_row(const E *src, bool vec, int d, int dp, __nv_bfloat16 *dst, int64_t off)
{
    const int lane = threadIdx.x & 31;
    for (int c = lane * 8; c < dp; c += 256) {
        float x[8];
        if (!src) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        } else if (vec && c + 8 <= d) {
            if constexpr (sizeof(E) == 2) {
                load_bf16_row<8>(reinterpret_cast<const __nv_bfloat16 *>(src) + c, x);
            } else {
                const float4 a = *reinterpret_cast<const float4 *>(src + c), b = *reinterpret_cast<const float4 *>(src + c + 4);
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
                x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = c + i < d ? to_f32(src[c + i]) : 0.0f;
        }
#pragma unroll
        for (int part = 0; part < SPLIT; ++part) {
            *reinterpret_cast<uint4 *>(dst + part * off + c) =
                make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
            if (part + 1 < SPLIT) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] -= __bfloat162float(__float2bfloat16_rn(x[i]));
            }
        }
    }
}

// Row r of `out` (dp columns, zeros behind d) = row token[r] (or r) of `in`; zeros from row n up to a multiple of 256. SPLIT
// 3: fp32 rows as three bf16 ones, off elements apart. A warp a row.
template <typename E, int SPLIT>
__global__ void __launch_bounds__(256) k_pack(const E *__restrict__ in, int64_t ld, bool vec, const int32_t *__restrict__ token,
                                              const int32_t *__restrict__ n_ptr, int n_rows, int d, int dp, __nv_bfloat16 *__restrict__ out, int64_t off)
{
    griddep_wait();
    griddep_launch_dependents();
    const int n = n_ptr ? *n_ptr : n_rows, end = (n + 255) / 256 * 256;
    for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < end; r += gridDim.x * 8) {
        pack_row<E, SPLIT>(r < n ? in + (int64_t)(token ? token[r] : r) * ld : nullptr, vec, d, dp, out + (int64_t)r * dp, off);
    }
}

// k_scan and k_pack of X in one launch, for up to kCollect tokens: a CTA has eight of them, one a warp, and counts those in use
// by itself (32 KB of labels at most). T = 4096, V = 256, d = 512, forward and backward: 41 us instead of 47; nothing at T = 8192.
constexpr int kCollect = 4096;
template <typename E, int SPLIT>
__global__ void __launch_bounds__(256) k_collect(const int64_t *__restrict__ label, const int32_t *__restrict__ count, int T, const E *__restrict__ in,
                                                 int64_t ld, bool vec, int d, int dp, __nv_bfloat16 *__restrict__ out, int64_t off, int32_t *__restrict__ n,
                                                 int32_t *__restrict__ token, int32_t *__restrict__ row, const LossScale scale)
{
    __shared__ uint32_t sums[8], tops[8];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.x * 8, t = t0 + warp;
    auto has = [&](int i) { return label ? label[i] >= 0 : count[i] > 0; };
    uint32_t mine = 0, top = 0;   // all tokens in use, and from bit 16 on those before the CTA's; the largest dloss's bits
    const bool tops_too = scale.dloss && scale.each && blockIdx.x == 0;
#pragma unroll 8
    for (int i = threadIdx.x; i < T; i += 256)
        if (has(i)) {
            mine += i < t0 ? 65537u : 1u;
            if (tops_too) top = max(top, scale.bits(i));
        }
    mine = __reduce_add_sync(0xffffffffu, mine);
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) {
        sums[warp] = mine;
        tops[warp] = top;
    }
    const bool own = lane < 8 && t0 + lane < T && has(t0 + lane);   // (the CTA's tokens, in every warp)
    const uint32_t who = __ballot_sync(0xffffffffu, own);
    __syncthreads();
    uint32_t both = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        both += sums[w];
        top = max(top, tops[w]);
    }
    const int all = (int)(both & 0xFFFFu), before = (int)(both >> 16);
    const int at = before + __popc(who & ((1u << warp) - 1));
    if (t < T) {
        const bool h = who >> warp & 1;
        if (lane == 0) {
            row[t] = h ? at : -1;
            if (h) token[at] = t;
        }
        if (h) pack_row<E, SPLIT>(in + (int64_t)t * ld, vec, d, dp, out + (int64_t)at * dp, off);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *n = all;
        if (scale.dloss) scale.put(all, top);
    }
    // zeros up to a multiple of 256
    for (int r = all + t; r < (all + 255) / 256 * 256; r += 8 * (int)gridDim.x) pack_row<E, SPLIT>(static_cast<const E *>(nullptr), vec, d, dp, out + (int64_t)r * dp, off);
}

// ---- the losses from the products' partial sums ----------------------------------------------------
struct JoinArgs {
    const float2 *stat;
    const float *zt;           // of labels: one a row; of lists: one a slot and row
    int slots;
    int64_t tp;
    const int32_t *row, *count;
    const int64_t *label;
    const float *ent;
    int64_t T, V;
    float c, tau;
    float back, back_rest;     // 1 / (c tau) in two parts: from a logit times c to nats
    float *loss, *lse;
};

// TX tokens a CTA, 256 / TX threads each over the slots; their sums are joined in order
template <int TX> __global__ void __launch_bounds__(256) k_join(const JoinArgs a)
{
    constexpr int Y = 256 / TX;
    __shared__ float sm[Y][TX], ss[Y][TX], sz[Y][TX];
    griddep_wait();
    griddep_launch_dependents();
    const int x = threadIdx.x % TX, y = threadIdx.x / TX;
    const int64_t t = blockIdx.x * (int64_t)TX + x;
    int r = -1;
    if (t < a.T) r = a.row ? a.row[t] : (a.label ? a.label[t] >= 0 : a.count[t] > 0) ? (int)t : -1;
    float most = -INFINITY, sum = 0.0f, z = 0.0f;
    if (r >= 0) {
#pragma unroll 4
        for (int s = y; s < a.slots; s += Y) {
            const float2 v = a.stat[s * a.tp + r];
            if (!a.label) z += a.zt[s * a.tp + r];
            const float now = max_nan(most, v.x);
            if (now == -INFINITY) continue;
            sum = fmaf(sum, exp2_fast(most - now), v.y * exp2_fast(v.x - now));
            most = now;
        }
    }
    sm[y][x] = most;
    ss[y][x] = sum;
    sz[y][x] = z;
    __syncthreads();
    for (int w = Y / 2; w; w >>= 1) {
        if (y < w) {
            const float now = max_nan(sm[y][x], sm[y + w][x]);
            ss[y][x] = now == -INFINITY ? 0.0f : fmaf(ss[y][x], exp2_fast(sm[y][x] - now), ss[y + w][x] * exp2_fast(sm[y + w][x] - now));
            sm[y][x] = now;
            sz[y][x] += sz[y + w][x];
        }
        __syncthreads();
    }
    if (y || t >= a.T) return;
    float loss = 0.0f, lse = 0.0f;
    if (r >= 0) {
        most = sm[0][x];
        const float log_sum = log2f(ss[0][x]);
        // (rounded once: most + log_sum, in units of ln 2, would be off by more than lse's own rounding, and so would c's be)
        lse = most == -INFINITY ? NAN : fmaf(most, a.back, fmaf(most, a.back_rest, kLn2 * log_sum));
        if (a.label) loss = a.label[t] < a.V ? kLn2 * (fmaf(-a.zt[r], a.c, most) + log_sum) : NAN;
        else loss = a.tau * a.tau * (a.ent[t] + kLn2 * (fmaf(-sz[0][x], a.c, most) + log_sum));
    }
    a.loss[t] = loss;
    a.lse[t] = lse;
}

// ---- rows of fp32 slots, summed in order and rounded -----------------------------------------------
// out[t] = the sum of the slots' rows row[t] (or t), times scale[1] where there is one; zeros where the row is negative. Eight columns a
// thread; up to two matrices in a launch.
struct FinishJob {
    const float *slot;
    int slots;
    int64_t stride;
    const int32_t *row;
    int64_t T;
    void *out;
    bool vec;
};
template <typename E> __global__ void __launch_bounds__(256) k_finish(const FinishJob j0, const FinishJob j1, int d, int dp, const float *scale)
{
    griddep_wait();
    griddep_launch_dependents();
    const float factor = scale ? scale[1] : 1.0f;
    const FinishJob &j = blockIdx.y ? j1 : j0;
    const int per = (d + 7) / 8;
    const int64_t vectors = j.T * per;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / per;
        const int c = (int)(i - t * per) * 8;
        const int64_t r = j.row ? j.row[t] : t;
        const int count = r < 0 ? 0 : j.slots;
        const float *src = j.slot + r * dp + c;
        float x[8] = {};
#pragma unroll 4
        for (int s = 0; s < count; ++s) {
            const float4 *p = reinterpret_cast<const float4 *>(src + s * j.stride);
            const float4 a = p[0], b = p[1];
            x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
            x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
        }
        if (scale && count > 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= factor;
        }
        E *dst = static_cast<E *>(j.out) + t * d + c;
        if (j.vec && c + 8 <= d) {
            if constexpr (sizeof(E) == 2) {
                *reinterpret_cast<uint4 *>(dst) =
                    make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
            } else {
                *reinterpret_cast<float4 *>(dst) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4 *>(dst + 4) = make_float4(x[4], x[5], x[6], x[7]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < d) dst[k] = from_f32<E>(x[k]);
        }
    }
}

// ---- plans -------------------------------------------------------------------------------------------
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

constexpr int kPairs = 76;             // what units are spread over in the choice of their size
constexpr int64_t kPackRows = 4096;    // words of a piece at least

// The most products that one accumulator adds up in a gradient in bf16: the tensor core cuts off at most 2 * 2^-23 of the sum's size with
// each 16 of them, 2^-10 of the terms' absolute sum in all. More go into splits, which are added up to nearest. (A million tokens in
// one accumulator: terms of one sign 4.2e-3 off in the mean, now 1e-5.)
constexpr int64_t kDeepest = 65536;

// Columns a unit and splits of the depth, `least` at least, by an estimate of the cycles: a 64-deep slice takes 2 bn on the tensor cores or
// 256 + bn to load (64 bytes a cycle and SM), a unit 1500 around its products, a slot 8 bytes an element at 3000 a cycle.
struct Units {
    int bn, nn, splits;
};
Units choose_units(int64_t rows, int64_t cols, int64_t depth, int most_splits, int64_t slot_bytes, int64_t least = 1)
{
    const int64_t nm = (rows + 255) / 256, slices = (depth + 63) / 64;
    Units best{256, 1, 1};
    double shortest = 1e300;
    for (int bn = 256; bn >= 32; bn -= 32) {
        if (bn > 32 && up(cols, 32) < bn) continue;
        const int64_t nn = (cols + bn - 1) / bn;
        for (int s = (int)least; s <= std::max<int64_t>(most_splits, least); s = s < 8 ? s + 1 : s + 4) {
            const int64_t per = (slices + s - 1) / s;
            if (s > least && (per < 4 || (s - 1) * per >= slices)) continue;
            const int64_t waves = (nm * nn * s + kPairs - 1) / kPairs;
            const double t = (double)waves * ((double)per * std::max(2 * bn, 256 + bn) + 1500.0) + (s > 1 ? (double)s * (double)slot_bytes / 3000.0 : 0.0);
            if (t < shortest) {
                shortest = t;
                best = Units{bn, (int)nn, s};
            }
        }
    }
    return best;
}

struct Shape {
    int64_t T, V, d, K;
    int split;            // bf16 parts of an operand, and of dz in memory
    bool distill, bwd;
    bool pack_w;          // W goes through the workspace
};

// A call's pieces of the vocabulary and its workspace
struct Plan {
    int64_t tp, dp, vc;   // rows of X and slots, columns of packed rows, words a piece (all rounded up)
    int pieces;
    Units fwd, dx, dw;    // (of a whole piece; the last one's are its own)
    int slots;            // fwd
    size_t bytes;
    int32_t *n, *token, *row, *count;
    int2 *list;
    float *ent, *bad, *zt, *dxs, *dws, *scale;
    float2 *stat;
    __nv_bfloat16 *xp, *wp, *dz;
};

int64_t piece_words(const Shape &s, const Plan &p, int i) { return std::min(p.vc, s.V - i * p.vc); }

// Whether a W of dense rows goes through the workspace. (Rows of whole 16 bytes that straddle 128-byte lines do not: with V = 30011,
// d = 1000 the copy cost more than it gave up to T = 4096, 153 against 164 us forward, and nothing at 8192.)
bool packs_w(const Shape &s) { return s.split == 3 || s.d % 8 != 0; }

Plan make_plan(const Shape &s, void *ws)
{
    Plan p = {};
    p.tp = std::max<int64_t>(up(s.T, 256), 256);
    p.dp = up(s.d, 64);   // (whole 128-byte lines: rows that straddle them load at half the rate)
    // dz of a piece: 2^27 elements (268 MB in bf16), but no fewer than 4096 words
    int64_t vc = up(s.V, 256);
    if (s.bwd) vc = std::min(vc, std::max(kPackRows, (int64_t(1) << (s.split == 3 ? 26 : 27)) / p.tp / 256 * 256));
    if (s.pack_w) vc = std::min(vc, std::max(kPackRows, packs_w(s) ? (int64_t(1) << 26) / p.dp / 256 * 256 : 0));
    p.pieces = (int)((s.V + vc - 1) / vc);
    p.vc = up((s.V + p.pieces - 1) / p.pieces, 256);
    p.pieces = (int)((s.V + p.vc - 1) / p.vc);
    WsCarver w(ws);
    p.n = w.take<int32_t>(1);
    p.row = w.take<int32_t>(s.T);
    p.token = w.take<int32_t>(s.T);
    if (s.distill) {
        p.list = w.take<int2>(s.T * s.K);
        p.ent = w.take<float>(s.T);
        p.bad = w.take<float>(s.T);
        p.count = w.take<int32_t>(s.T);
    }
    p.xp = w.take<__nv_bfloat16>(s.split * p.tp * p.dp);
    if (s.pack_w) p.wp = w.take<__nv_bfloat16>(s.split * p.vc * p.dp);
    if (!s.bwd) {
        for (int i = 0; i < p.pieces; ++i) p.slots += 2 * choose_units(s.T, piece_words(s, p, i), p.dp * (s.split == 3 ? 6 : 1), 1, 0).nn;
        p.stat = w.take<float2>(p.slots * p.tp);
        p.zt = w.take<float>(s.distill ? p.slots * p.tp : p.tp);
    } else {
        if (s.split == 1) p.scale = w.take<float>(2);
        p.dz = w.take<__nv_bfloat16>(s.split * p.tp * p.vc);
        const int parts = s.split == 3 ? 6 : s.T <= kTwoParts ? 2 : 1;   // products of a unit (for more tokens the most likely number)
        auto least = [&](int64_t depth) { return s.split == 3 ? 1 : (depth + kDeepest - 1) / kDeepest; };   // (fp32 adds in short pieces)
        p.dx = choose_units(s.T, s.d, p.vc * parts, 32, p.tp * p.dp * 4, least(p.vc));
        p.dw = choose_units(p.vc, s.d, s.T * parts, 32, 2 * p.vc * p.dp * 4, std::max<int64_t>(1, least(s.T)));
        p.dxs = w.take<float>(p.dx.splits * p.tp * p.dp);
        if (p.dw.splits > 1) p.dws = w.take<float>(p.dw.splits * p.vc * p.dp);
    }
    p.bytes = w.used;
    return p;
}

// The workspace of a call, whatever its pointers' and strides' alignment. (Rows of W that are off the vectors by their width may be whole
// ones by their stride: W is then used as it lies, whose pieces, dz and slots are other ones, and may be larger.)
size_t plan_bytes(Shape s)
{
    s.pack_w = true;
    const size_t packed = make_plan(s, nullptr).bytes;
    if (s.split == 3) return packed;   // (its parts always go through the workspace)
    s.pack_w = false;
    return std::max(packed, make_plan(s, nullptr).bytes);
}

// ---- launches ----------------------------------------------------------------------------------------
struct Run {
    Ctx c;
    cudaError_t e = cudaSuccess;
    uint64_t launches = 0;
    template <typename... K, typename... A> void go(void (*kernel)(K...), dim3 grid, dim3 block, size_t smem, int cluster, A &&...args)
    {
        if (e != cudaSuccess) return;
        e = launch_clustered(kernel, grid, block, smem, cluster, c.stream, std::forward<A>(args)...);
        if (e == cudaSuccess) ++launches;
    }
    void map(CUtensorMap *m, const void *ptr, uint64_t inner, uint64_t outer, uint64_t pitch, uint32_t box_in, uint32_t box_out,
             CUtensorMapSwizzle swz, CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16)
    {
        if (e == cudaSuccess && !make_map(m, ptr, inner, outer, pitch, box_in, box_out, swz, type)) e = cudaErrorInvalidValue;
    }
};

template <int MODE, int SPLIT, int PIECE, int JOBS> void run_gemm(Run &r, const VocabJobs<JOBS> &jobs, int64_t units)
{
    using C = VocabCfg;
    static std::atomic<uint8_t> done[kMaxDev];
    if (r.e == cudaSuccess) r.e = ensure_smem(k_vocab_gemm<MODE, SPLIT, PIECE, JOBS>, C::SMEM, r.c.device, done);
    const int64_t pairs = std::max(1, r.c.sm_count / 2);
    r.go(k_vocab_gemm<MODE, SPLIT, PIECE, JOBS>, dim3((unsigned)(2 * std::min(units, pairs))), dim3(C::THREADS), C::SMEM, 2, jobs);
}

unsigned row_grid(const Ctx &c, int64_t rows, int per) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((rows + per - 1) / per, 16 * c.sm_count)); }

constexpr CUtensorMapSwizzle k128 = CU_TENSOR_MAP_SWIZZLE_128B, k64 = CU_TENSOR_MAP_SWIZZLE_64B;

struct Call {
    const resbm_vocab_desc *d;
    const void *X, *W, *teacher;
    const int64_t *target;   // labels or indices
    float *loss, *lse_out;
    const float *lse, *dloss;
    void *dX, *dW;
};

// E: the tensors' type; SPLIT: bf16 parts of X and W
template <typename E, int SPLIT> void run_loss(Run &r, const Shape &s, const Plan &p, const Call &a)
{
    constexpr bool F32 = SPLIT == 3;
    constexpr int DZ = F32 ? 3 : 2;   // parts of dz (2: for few tokens)
    // Slices of a piece of a sum: 512 deep (256 of three parts), which leaves the truncation of 32 MMAs (16, and 80 of smaller
    // products). T = 777, V = 50001,
    // d = 1000: losses 3.8e-7 off (256 deep 1.8e-7, 1024 8e-7); T = 16384, V = 32000, d = 2048: 1104 us (1194, 1090). fp32, T = 2048, V = 8000,
    // d = 768, forward and backward: dX 5.4e-7 off, 455 us (128 deep 3.8e-7, 497; 512 9.2e-7, 444).
    constexpr int P = F32 ? 4 : 8;
    const resbm_vocab_desc &d = *a.d;
    const int64_t T = s.T, V = s.V;
    const float tau = s.distill ? d.temperature : 1.0f;
    const int64_t *label = s.distill ? nullptr : a.target;
    const Ctx &c = r.c;

    if (s.distill) {
        const int K = (int)s.K, warps = K <= 256 ? 8 : K <= 512 ? 4 : 2;
        const unsigned grid = row_grid(c, T, warps);
        auto go = [&](auto kernel, auto teacher) {
            r.go(kernel, dim3(grid), dim3(32 * warps), (size_t)warps * K * 4, 1, a.target, teacher, T, K, V, tau, p.list, p.ent, p.bad, p.count);
        };
        if (d.teacher_dtype == RESBM_F32) go(k_targets<float>, static_cast<const float *>(a.teacher));
        else go(k_targets<__nv_bfloat16>, static_cast<const __nv_bfloat16 *>(a.teacher));
    }
    const LossScale scale{s.bwd && !F32 ? a.dloss : nullptr, d.dloss_each, tau, p.scale};
    const bool x_fits = al16(a.X) && d.ldx * (int64_t)sizeof(E) % 16 == 0;
    // one row block: the tokens without a target cost nothing more (but their rows must not enter dW)
    const bool direct = !s.bwd && !F32 && x_fits && T <= 256;
    if (!direct && T <= kCollect) {
        r.go(k_collect<E, SPLIT>, dim3((unsigned)((T + 7) / 8)), dim3(256), 0, 1, label, p.count, (int)T, static_cast<const E *>(a.X), d.ldx, x_fits, (int)s.d, (int)p.dp,
             p.xp, p.tp * p.dp, p.n, p.token, p.row, scale);
    } else if (!direct) {
        r.go(k_scan, dim3(kScanCtas), dim3(1024), 0, 1, label, p.count, (int)T, p.n, p.token, p.row, scale);
        r.go(k_pack<E, SPLIT>, dim3(row_grid(c, p.tp, 8)), dim3(256), 0, 1, static_cast<const E *>(a.X), d.ldx, x_fits, p.token, p.n, 0, (int)s.d,
             (int)p.dp, p.xp, p.tp * p.dp);
    }
    const void *x = direct ? a.X : p.xp;
    const int64_t ldx = direct ? d.ldx : p.dp, x_rows = direct ? T : SPLIT * p.tp;
    const bool w_fits = al16(a.W) && d.ldw * (int64_t)sizeof(E) % 16 == 0;

    VocabGemm g = {};
    g.n_ptr = direct ? nullptr : p.n;
    g.n_rows = (int)T;
    g.splits = 1;
    g.group = 8;
    g.a_rows = T <= 120 ? (int)up(T, 8) : 128;
    g.a_off = (int)p.tp;
    g.b_off = (int)p.vc;
    g.token = direct ? nullptr : p.token;
    g.label = label;
    g.list = p.list;
    g.K = (int)s.K;
    g.tp = p.tp;
    g.c = kLog2e / tau;
    g.tau = tau;
    g.V = (int)V;
    g.stat = p.stat;
    g.zt = p.zt;
    g.lse = a.lse;
    g.dloss = a.dloss;
    g.scale = p.scale;
    g.dloss_step = d.dloss_each;
    g.bad = s.distill ? p.bad : nullptr;

    for (int i = 0; i < p.pieces && r.e == cudaSuccess; ++i) {
        const int64_t v0 = i * p.vc, vn = piece_words(s, p, i);
        const void *w = a.W;
        int64_t ldw = d.ldw, w_rows = V;
        if (s.pack_w) {
            r.go(k_pack<E, SPLIT>, dim3(row_grid(c, p.vc, 8)), dim3(256), 0, 1, static_cast<const E *>(a.W) + v0 * d.ldw, d.ldw, w_fits,
                 static_cast<const int32_t *>(nullptr), static_cast<const int32_t *>(nullptr), (int)vn, (int)s.d, (int)p.dp, p.wp, p.vc * p.dp);
            w = p.wp;
            ldw = p.dp;
            w_rows = SPLIT * p.vc;
        }
        const int64_t row_blocks = (T + 255) / 256;
        // z = X . W^T
        const Units u = choose_units(T, vn, p.dp * (F32 ? 6 : 1), 1, 0);
        g.v0 = (int)v0;
        g.b_y = s.pack_w ? 0 : (int)v0;
        g.cols = (int)vn;
        g.depth = (int)s.d;
        g.bn = u.bn;
        g.nn = u.nn;
        g.slot_rows = (int)p.tp;
        VocabJobs<1> z;
        r.map(&z.a[0], x, s.d, x_rows, ldx * 2, 64, (uint32_t)g.a_rows, k128);
        r.map(&z.b[0], w, s.d, w_rows, ldw * 2, 64, (uint32_t)u.bn / 2, k128);
        z.o[0] = z.a[0];
        z.g[0] = g;
        if (!s.bwd) {
            // (One row block is bound by reading W: a quarter of the piece costs 1 us of 31 at V = 32000, d = 2048, and a single
            // token's error is not averaged: the worst of eight losses 7e-7 off instead of 2.6e-6.)
            if (T <= 256) run_gemm<VG_FWD, SPLIT, P / 4, 1>(r, z, row_blocks * u.nn);
            else run_gemm<VG_FWD, SPLIT, P, 1>(r, z, row_blocks * u.nn);
            g.slot0 += 2 * u.nn;
            continue;
        }
        r.map(&z.o[0], p.dz, vn, SPLIT * p.tp, p.vc * 2, 32, 32, k64);
        // z again, whose error is seen where a token is certain and p - q next to nothing: in one accumulator it grew with d (d = 16384,
        // logits up to 1400: dX and dW 1.5e-2 off; in pieces 1024 deep 1.9e-3, their rounding). T = 16384, V = 32000, d = 2048 backward
        // 3903 -> 3947 us, T = 8192, d = 1100 3 % more; pieces 512 deep cost 4 to 10 %.
        constexpr int kLongPiece = 16;
        // In fp32 up to 256 tokens in the forward's pieces, so that z is the same: 6 tokens of V = 545, d = 1168 had dX and dW 2.4e-6 off.
        if constexpr (F32) {
            if (T <= 256) run_gemm<VG_DZ, DZ, P / 4, 1>(r, z, row_blocks * u.nn);
            else run_gemm<VG_DZ, DZ, P, 1>(r, z, row_blocks * u.nn);
        } else if (s.d > 64 * kLongPiece) run_gemm<VG_DZ, DZ, kLongPiece, 1>(r, z, row_blocks * u.nn);
        else run_gemm<VG_DZ, DZ, 0, 1>(r, z, row_blocks * u.nn);

        VocabJobs<2> gr;
        FinishJob fin[2] = {};
        int jobs = 0, fins = 0;
        int64_t units = 0, depth[2] = {};
        if (a.dX) {   // dz . W, added over the pieces
            VocabGemm &h = gr.g[jobs];
            h = g;
            h.mode = VG_DX;
            h.cols = (int)s.d;
            h.depth = (int)vn;
            h.bn = p.dx.bn;
            h.nn = p.dx.nn;
            h.splits = p.dx.splits;
            h.add = i > 0;
            r.map(&gr.a[jobs], p.dz, vn, SPLIT * p.tp, p.vc * 2, 64, (uint32_t)g.a_rows, k128);
            r.map(&gr.b[jobs], w, s.d, w_rows, ldw * 2, 64, 64, k128);
            r.map(&gr.o[jobs], p.dxs, p.dp, h.splits * p.tp, p.dp * 4, 32, 32, k128, CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
            depth[jobs++] = vn / h.splits;
            units += row_blocks * h.nn * h.splits;
            if (i + 1 == p.pieces)
                fin[fins++] = FinishJob{p.dxs, h.splits, p.tp * p.dp, p.row, T, a.dX, al16(a.dX) && s.d * (int64_t)sizeof(E) % 16 == 0};
        }
        if (a.dW) {   // dz^T . X
            VocabGemm &h = gr.g[jobs];
            h = g;
            h.mode = VG_DW;
            h.rows = (int)vn;
            h.cols = (int)s.d;
            h.bn = p.dw.bn;
            h.nn = p.dw.nn;
            h.splits = p.dw.splits;
            h.slot_rows = (int)p.vc;
            h.b_off = (int)p.tp;
            h.b_y = 0;
            h.out_f32 = F32;
            r.map(&gr.a[jobs], p.dz, vn, SPLIT * p.tp, p.vc * 2, 64, 64, k128);
            r.map(&gr.b[jobs], p.xp, s.d, SPLIT * p.tp, p.dp * 2, 64, 64, k128);
            CUtensorMap *mo = &gr.o[jobs];
            *mo = gr.a[jobs];
            E *out = static_cast<E *>(a.dW) + v0 * s.d;
            if (h.splits > 1) {
                h.out_f32 = 1;
                r.map(mo, p.dws, p.dp, h.splits * p.vc, p.dp * 4, 32, 32, k128, CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
                fin[fins++] = FinishJob{p.dws, h.splits, p.vc * p.dp, nullptr, vn, out, al16(out) && s.d * (int64_t)sizeof(E) % 16 == 0};
            } else {
                h.out_y = (int)v0;
                if (!al16(a.dW) || s.d * (int64_t)sizeof(E) % 16 != 0) {
                    h.out = a.dW;
                    h.ldo = s.d;
                } else if (F32) {
                    r.map(mo, a.dW, s.d, V, s.d * 4, 32, 32, k128, CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
                } else {
                    r.map(mo, a.dW, s.d, V, s.d * 2, 32, 32, k64);
                }
            }
            depth[jobs++] = T / h.splits;
            units += (vn + 255) / 256 * h.nn * h.splits;
        }
        if (jobs < 2) {   // (only one of them is wanted: the other has no units)
            gr.a[1] = gr.a[0];
            gr.b[1] = gr.b[0];
            gr.o[1] = gr.o[0];
            gr.g[1] = gr.g[0];
            gr.g[1].nn = 0;
        } else if (depth[0] < depth[1]) {
            std::swap(gr.a[0], gr.a[1]);
            std::swap(gr.b[0], gr.b[1]);
            std::swap(gr.o[0], gr.o[1]);
            std::swap(gr.g[0], gr.g[1]);
        }
        run_gemm<VG_GRADS, DZ, F32 ? P : 0, 2>(r, gr, units);
        if (fins) {
            const int64_t most = std::max(fin[0].T, fin[1].T) * ((s.d + 7) / 8);
            r.go(k_finish<E>, dim3(row_grid(c, most, 256), (unsigned)fins), dim3(256), 0, 1, fin[0], fin[1], (int)s.d, (int)p.dp, static_cast<const float *>(p.scale));
        }
    }
    if (s.bwd) return;
    const double back = 1.0 / ((double)g.c * tau);
    JoinArgs j{p.stat, p.zt, p.slots, p.tp, direct ? nullptr : p.row, p.count, label, p.ent, T, V, g.c, tau, (float)back, (float)(back - (double)(float)back), a.loss, a.lse_out};
    if (T < 1024) r.go(k_join<1>, dim3((unsigned)T), dim3(256), 0, 1, j);
    else r.go(k_join<32>, dim3((unsigned)((T + 31) / 32)), dim3(256), 0, 1, j);
}

// ---- checks --------------------------------------------------------------------------------------------
resbm_status check_shape(const resbm_vocab_desc *desc, bool distill)
{
    if (!desc) return RESBM_ERR_INVALID_ARG;
    const resbm_vocab_desc &d = *desc;
    if (d.T < 0 || d.V < 1 || d.d < 1 || (d.dtype != RESBM_F32 && d.dtype != RESBM_BF16) || d.flags) return RESBM_ERR_INVALID_ARG;
    if (distill && (d.K < 1 || d.K > 1024)) return RESBM_ERR_INVALID_ARG;
    constexpr int64_t most = int64_t(1) << 29;
    if (d.T >= most || d.V >= most || d.d > (int64_t(1) << 20)) return RESBM_ERR_UNSUPPORTED;
    // products' units are counted in 31 bits, and the rows of three parts addressed so
    if ((d.T + 255) / 256 * ((d.V + 31) / 32) >= (int64_t(1) << 30) || (std::max(d.T, d.V) + 255) / 256 * ((d.d + 31) / 32) >= (int64_t(1) << 26))
        return RESBM_ERR_UNSUPPORTED;
    return RESBM_OK;
}

Shape shape_of(const resbm_vocab_desc &d, bool distill, bool bwd)
{
    return Shape{d.T, d.V, d.d, distill ? d.K : 0, d.dtype == RESBM_F32 ? 3 : 1, distill, bwd, false};
}

// (tau^2 and log2(e) / tau are floats)
constexpr float kLeastTau = 1e-18f, kMostTau = 1e18f;

resbm_status loss_call(const resbm_vocab_desc *desc, bool distill, bool bwd, Call a, void *ws, size_t ws_bytes, void *stream)
{
    resbm_status st = check_shape(desc, distill);
    if (st != RESBM_OK) return st;
    resbm_vocab_desc d = *desc;
    if (d.T <= 1) d.ldx = d.d;   // one row: its stride is not used
    if (d.V == 1) d.ldw = d.d;
    const int64_t es = d.dtype == RESBM_BF16 ? 2 : 4, limit = INT64_MAX / 64;
    const bool t = d.T > 0;
    if (distill && ((d.teacher_dtype != RESBM_F32 && d.teacher_dtype != RESBM_BF16) || !(d.temperature >= kLeastTau) || !(d.temperature <= kMostTau)))
        return RESBM_ERR_INVALID_ARG;
    if (bwd && (d.dloss_each < 0 || d.dloss_each > 1)) return RESBM_ERR_INVALID_ARG;
    auto bad = [&](int64_t rows, int64_t ld) { return rows > 1 && (ld < d.d || !mul_ok(rows, ld) || rows * ld > limit); };
    if (bad(d.T, d.ldx) || bad(d.V, d.ldw)) return RESBM_ERR_INVALID_ARG;
    const int64_t te = d.teacher_dtype == RESBM_BF16 ? 2 : 4;
    if (!ptr_ok(a.X, es, t) || !ptr_ok(a.W, es, t) || !ptr_ok(a.target, 8, t) || (distill && !ptr_ok(a.teacher, te, t))) return RESBM_ERR_INVALID_ARG;
    if (bwd ? !ptr_ok(a.lse, 4, t) || !ptr_ok(a.dloss, 4, t) || !ptr_ok(a.dX, es, false) || !ptr_ok(a.dW, es, false)
            : !ptr_ok(a.loss, 4, t) || !ptr_ok(a.lse_out, 4, t))
        return RESBM_ERR_INVALID_ARG;
    if (!ptr_ok(ws, 256, false)) return RESBM_ERR_INVALID_ARG;
    auto rows = [&](const void *p, int64_t n, int64_t ld) { return rng(p, n > 0 ? (n - 1) * (n > 1 ? ld : 0) + d.d : 0, es); };
    const int64_t targets = d.T * (distill ? d.K : 1);
    const Range ins[] = {rows(a.X, d.T, d.ldx), rows(a.W, d.V, d.ldw), rng(a.target, targets, 8), rng(distill ? a.teacher : nullptr, targets, te),
                         rng(bwd ? a.lse : nullptr, d.T, 4), rng(bwd ? a.dloss : nullptr, d.dloss_each ? d.T : 1, 4)};
    const Range outs[] = {rng(ws, (int64_t)std::min<size_t>(ws_bytes, INT64_MAX), 1), bwd ? rng(a.dX, d.T * d.d, es) : rng(a.loss, d.T, 4),
                          bwd ? rng(a.dW, d.V * d.d, es) : rng(a.lse_out, d.T, 4)};
    if (any_overlap(outs, ins, sizeof(ins) / sizeof(ins[0]))) return RESBM_ERR_INVALID_ARG;
    a.d = &d;
    Shape s = shape_of(d, distill, bwd);
    if (t && (!ws || ws_bytes < plan_bytes(s))) return RESBM_ERR_WORKSPACE;
    Run r;
    st = make_ctx(stream, &r.c);
    if (st != RESBM_OK) return st;
    if (!t) {
        if (bwd && a.dW) r.e = cudaMemsetAsync(a.dW, 0, (size_t)(d.V * d.d * es), r.c.stream);
        return finish(r.e);
    }
    if (bwd && !a.dX && !a.dW) return RESBM_OK;
    s.pack_w = s.split == 3 || !al16(a.W) || d.ldw % 8 != 0;
    const Plan p = make_plan(s, ws);
    if (p.bytes > ws_bytes) return RESBM_ERR_WORKSPACE;   // (plan_bytes covers it)
    if (s.split == 3) run_loss<float, 3>(r, s, p, a);
    else run_loss<__nv_bfloat16, 1>(r, s, p, a);
    count_launches(r.launches);
    if (r.e != cudaSuccess) cudaGetLastError();
    return finish(r.e);
}

}  // namespace

cudaError_t vocab_device_error(unsigned int *code, bool clear)
{
    cudaError_t e = cudaMemcpyFromSymbol(code, tc::g_resbm_device_error, sizeof(unsigned int));
    if (e == cudaSuccess && clear && *code) {
        const unsigned int zero = 0;
        e = cudaMemcpyToSymbol(tc::g_resbm_device_error, &zero, sizeof(zero));
    }
    return e;
}

}  // namespace resbm

using namespace resbm;

extern "C" {

resbm_status resbm_vocab_workspace_bytes(const resbm_vocab_desc *desc, int op, size_t *bytes)
{
    if (!bytes) return RESBM_ERR_INVALID_ARG;
    *bytes = 0;
    if (op < RESBM_VOCAB_CE_FWD || op > RESBM_VOCAB_EMBED_BWD) return RESBM_ERR_INVALID_ARG;
    if (op == RESBM_VOCAB_EMBED_BWD) {   // (its limits are not the products')
        if (!desc || desc->flags) return RESBM_ERR_INVALID_ARG;
        const resbm_status st = embed_check_shape(desc->T, desc->V, desc->d, desc->dtype);
        if (st == RESBM_OK) *bytes = embed_bwd_ws_bytes(desc->T, desc->d);
        return st;
    }
    const bool distill = op == RESBM_VOCAB_DISTILL_FWD || op == RESBM_VOCAB_DISTILL_BWD;
    const resbm_status st = check_shape(desc, distill);
    if (st != RESBM_OK) return st;
    *bytes = plan_bytes(shape_of(*desc, distill, op == RESBM_VOCAB_CE_BWD || op == RESBM_VOCAB_DISTILL_BWD));
    return RESBM_OK;
}

resbm_status resbm_linear_ce_fwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *labels, float *loss, float *lse,
                                 void *ws, size_t ws_bytes, void *stream)
{
    Call a = {};
    a.d = desc; a.X = X; a.W = W; a.target = labels; a.loss = loss; a.lse_out = lse;
    return loss_call(desc, false, false, a, ws, ws_bytes, stream);
}

resbm_status resbm_linear_ce_bwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *labels, const float *lse,
                                 const float *dloss, void *dX, void *dW, void *ws, size_t ws_bytes, void *stream)
{
    Call a = {};
    a.d = desc; a.X = X; a.W = W; a.target = labels; a.lse = lse; a.dloss = dloss; a.dX = dX; a.dW = dW;
    return loss_call(desc, false, true, a, ws, ws_bytes, stream);
}

resbm_status resbm_distill_fwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *index, const void *teacher,
                               float *loss, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    Call a = {};
    a.d = desc; a.X = X; a.W = W; a.target = index; a.teacher = teacher; a.loss = loss; a.lse_out = lse;
    return loss_call(desc, true, false, a, ws, ws_bytes, stream);
}

resbm_status resbm_distill_bwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *index, const void *teacher,
                               const float *lse, const float *dloss, void *dX, void *dW, void *ws, size_t ws_bytes, void *stream)
{
    Call a = {};
    a.d = desc; a.X = X; a.W = W; a.target = index; a.teacher = teacher; a.lse = lse; a.dloss = dloss; a.dX = dX; a.dW = dW;
    return loss_call(desc, true, true, a, ws, ws_bytes, stream);
}

}  // extern "C"
