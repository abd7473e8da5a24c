// embed.cu -- resbm_embed_fwd and resbm_embed_bwd (include/resbm_vocab.h): rows of a table times a scale, and the table's
// gradient from tokens sorted by id.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "abi.h"
#include "common.cuh"
#include "resbm_vocab.h"
#include "tc_host.cuh"
#include "vocab.h"

namespace resbm {
namespace {

// A thread's columns of a row as fp32: VEC neighbours (16 bytes), or off the 16-byte grid (STEP > 0) VEC single ones STEP apart
template <typename E, int VEC, int STEP> struct Cols {
    float x[VEC];
    // left: columns from p on that exist
    __device__ __forceinline__ void load(const E *p, int64_t left)
    {
        if constexpr (STEP > 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = i * STEP < left ? to_f32(__ldg(p + i * STEP)) : 0.0f;
        } else {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(E) == 2) {
                    x[2 * i] = __uint_as_float(w[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                } else {
                    x[i] = __uint_as_float(w[i]);
                }
            }
        }
    }
    __device__ __forceinline__ void store(E *p, int64_t left, float scale) const
    {
        if constexpr (STEP > 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i * STEP < left) p[i * STEP] = from_f32<E>(x[i] * scale);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(E) == 2) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i] * scale, x[2 * i + 1] * scale);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                } else {
                    w[i] = __float_as_uint(x[i] * scale);
                }
            }
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // fp32 partial sums (rows of whole vectors where STEP is 0)
    __device__ __forceinline__ void put(float *p, int64_t left) const
    {
        if constexpr (STEP > 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i * STEP < left) p[i * STEP] = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        }
    }
    __device__ __forceinline__ void get(const float *p, int64_t left)
    {
        if constexpr (STEP > 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = i * STEP < left ? p[i * STEP] : 0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(p + i);
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ void fill(float v)
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = v;
    }
    __device__ __forceinline__ void add(const Cols &o)
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] += o.x[i];
    }
};

// The columns of a thread: 2^log_tx threads along a row, those of blockIdx.y
template <int VEC, int STEP> __device__ __forceinline__ int64_t first_col(int log_tx)
{
    const int x = threadIdx.x & ((1 << log_tx) - 1);
    if (STEP) return (int64_t)blockIdx.y * (VEC * STEP) + x;   // (STEP threads along a row)
    return (((int64_t)blockIdx.y << log_tx) + x) * VEC;
}

// ---- forward -----------------------------------------------------------------------------------------
// 2^log_tx threads along a row, 256 >> log_tx rows a CTA at a time, four rows in flight a thread
template <typename E, int VEC, int STEP>
__global__ void __launch_bounds__(256) k_embed_fwd(const int64_t *__restrict__ ids, const E *__restrict__ table, int64_t ldt, E *__restrict__ out,
                                                   int64_t ldo, int64_t T, int64_t V, int64_t d, float scale, int log_tx)
{
    griddep_wait();
    griddep_launch_dependents();
    const int64_t col = first_col<VEC, STEP>(log_tx), left = d - col;
    if (left <= 0) return;
    const int rows = 256 >> log_tx;
    const int64_t step = (int64_t)gridDim.x * rows;
    for (int64_t t = (int64_t)blockIdx.x * rows + (threadIdx.x >> log_tx); t < T; t += 4 * step) {
        int64_t id[4];
        Cols<E, VEC, STEP> v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = t + i * step < T ? ids[t + i * step] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (id[i] >= 0 && id[i] < V) v[i].load(table + id[i] * ldt + col, left);
            else v[i].fill(NAN);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i * step < T) v[i].store(out + (t + i * step) * ldo + col, left, scale);
    }
}

// ---- tokens sorted by id -------------------------------------------------------------------------------
constexpr int kZeroClusters = 13, kSortCtas = 8, kSortThreads = 1024, kMaxBins = 512;

// The first cluster sorts, the others write zeros over dtable meanwhile: most words have no tokens, and the sums
// overwrite the rows of those that have (16384 tokens of 32000 words: 22 MB of 131).
//
// Stable: one cluster of eight CTAs, a radix sort of the ids from their lowest digit on. Each warp has a contiguous run of the
// positions; its equal digits are found 32 at a time by a match, so that ranks need no atomics and keep the order. Ids that
// count for nothing become V and sort behind the others. T = 16384 tokens of 32000 words are two passes of 8 bits. (A sort over the whole GPU would be several launches; this one's time is their latency.)
__global__ void __cluster_dims__(kSortCtas) __launch_bounds__(kSortThreads, 1)
    k_sort(const int64_t *__restrict__ ids, int T, int V, int64_t padding, int passes, int bits, int32_t *keys, int32_t *vals, uint8_t *dtable, int64_t bytes)
{
    extern __shared__ __align__(128) int32_t cnt[];   // 32 warps x bins: counts, then places
    __shared__ int32_t total[kMaxBins], wsum[32];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    if (cluster_index() > 0) {
        // (bulk copies out of shared memory: plain 16-byte stores of these CTAs reached 4.6 TB/s)
        constexpr int64_t chunk = 32768;
        const int64_t head = min((int64_t)((16 - (reinterpret_cast<uintptr_t>(dtable) & 15)) & 15), bytes), body = (bytes - head) / 16 * 16;
        const int64_t first = blockIdx.x - kSortCtas, step = gridDim.x - kSortCtas;
        for (int i = tid; i < chunk / 16; i += kSortThreads) reinterpret_cast<uint4 *>(cnt)[i] = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            for (int64_t at = first * chunk; at < body; at += step * chunk) {
                const uint32_t size = (uint32_t)(body - at < chunk ? body - at : chunk);
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dtable + head + at), "r"(smem_addr(cnt)), "r"(size) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 4;" ::: "memory");
            }
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
        if (first == 0 && tid >= 32 && tid < 32 + head) dtable[tid - 32] = 0;
        if (first == 0 && tid >= 64 && tid < 64 + bytes - head - body) dtable[head + body + tid - 64] = 0;
        return;
    }
    const int rank = (int)cluster_rank(), bins = 1 << bits;
    const int per_warp = ((T + kSortCtas * 32 - 1) / (kSortCtas * 32) + 31) / 32 * 32;
    const int64_t first = ((int64_t)rank * 32 + warp) * per_warp;
    const int p0 = (int)(first < T ? first : T), p1 = (int)(first + per_warp < T ? first + per_warp : T);
    int32_t *mine = cnt + warp * bins;
    for (int pass = 0; pass < passes; ++pass) {
        const int32_t *kin = keys + (int64_t)((pass & 1) ^ 1) * T, *vin = vals + (int64_t)((pass & 1) ^ 1) * T;
        int32_t *kout = keys + (int64_t)(pass & 1) * T, *vout = vals + (int64_t)(pass & 1) * T;
        const int shift = pass * bits;
        auto key_at = [&](int p) -> int32_t {
            if (pass) return __ldcg(kin + p);
            const int64_t id = ids[p];
            return id < 0 || id >= V || id == padding ? V : (int32_t)id;
        };
        for (int b = lane; b < bins; b += 32) mine[b] = 0;
        __syncwarp();
        for (int p = p0; p < p1; p += 32) {
            const bool in = p + lane < p1;
            const int digit = in ? (key_at(p + lane) >> shift) & (bins - 1) : bins;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            if (in && (same & ((1u << lane) - 1)) == 0) mine[digit] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // counts -> places within the CTA's tokens of a digit; total[b]: the CTA's
        if (tid < bins) {
            int sum = 0;
            for (int w = 0; w < 32; ++w) {
                const int v = cnt[w * bins + tid];
                cnt[w * bins + tid] = sum;
                sum += v;
            }
            total[tid] = sum;
        }
        cluster_sync();
        int all = 0, before = 0;   // digit tid: over all CTAs, over those before this one
        if (tid < bins) {
            for (int c = 0; c < kSortCtas; ++c) {
                int v;
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(map_shared(smem_addr(&total[tid]), (uint32_t)c)));
                all += v;
                if (c < rank) before += v;
            }
        }
        int upto = all;   // inclusive sum over the digits
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) wsum[warp] = upto;
        __syncthreads();
        for (int w = 0; w < warp; ++w) upto += wsum[w];
        if (tid < bins)
            for (int w = 0; w < 32; ++w) cnt[w * bins + tid] += upto - all + before;
        __syncthreads();
        for (int p = p0; p < p1; p += 32) {
            const bool in = p + lane < p1;
            const int32_t key = in ? key_at(p + lane) : 0;
            const int digit = in ? (key >> shift) & (bins - 1) : bins;
            const uint32_t same = __match_any_sync(0xffffffffu, digit), below = same & ((1u << lane) - 1);
            const int at = in ? mine[digit] + __popc(below) : 0;
            __syncwarp();
            if (in) {
                if (below == 0) mine[digit] += __popc(same);
                __stcg(kout + at, key);
                __stcg(vout + at, pass ? __ldcg(vin + p + lane) : p + lane);
            }
            __syncwarp();
        }
        __threadfence();
        cluster_sync();   // (and no CTA reads another's totals any more)
    }
}

// ---- sums ------------------------------------------------------------------------------------------------
constexpr int kRun = 32;   // sorted positions a block

struct SumArgs {
    const int32_t *keys, *vals;   // sorted
    const void *dout;
    void *dtable;
    float *part;                  // (block, head or tail, column)
    int64_t ldo, d;
    int T, V, log_tx;
    float scale;
};

// Blocks of kRun sorted positions, 2^log_tx threads along a row, which add the rows of each word up in order, sixteen in
// flight. A word whose tokens all lie in the block is finished; the block's first and last runs may be pieces of longer ones, and
// leave a partial sum. So this kernel's work is even whatever the ids are; k_embed_join's is not: a word on half of 65536 tokens is
// 1024 partial rows, added up by the threads of one block.
template <typename E, int VEC, int STEP> __global__ void __launch_bounds__(256, 3) k_embed_sum(const SumArgs a)
{
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t b = (int64_t)blockIdx.x * (256 >> a.log_tx) + (threadIdx.x >> a.log_tx);   // (the same for a warp)
    const int64_t col = first_col<VEC, STEP>(a.log_tx), left = a.d - col;
    const int64_t p0 = b * kRun;
    if (p0 >= a.T) return;
    const int len = a.T - p0 < kRun ? (int)(a.T - p0) : kRun;
    // the block's keys and tokens, one a lane
    const int32_t k = lane < len ? a.keys[p0 + lane] : a.V, tok = lane < len ? a.vals[p0 + lane] : 0;
    const int32_t before = p0 > 0 ? a.keys[p0 - 1] : -1, after = p0 + len < a.T ? a.keys[p0 + len] : -1;
    const bool head = __shfl_sync(0xffffffffu, k, 0) == before;          // the first run began before
    const bool tail = __shfl_sync(0xffffffffu, k, len - 1) == after;     // the last one goes on
    const int used = __popc(__ballot_sync(0xffffffffu, k < a.V));        // (keys ascend)
    const E *dout = static_cast<const E *>(a.dout) + col;
    float *part = a.part + b * 2 * a.d + col;
    constexpr int F = STEP ? 4 : 32 / VEC;   // rows in flight
    Cols<E, VEC, STEP> sum;
    sum.fill(0.0f);
    bool first_run = true;
#pragma unroll 1
    for (int i = 0; i < used; i += F) {
        Cols<E, VEC, STEP> v[F];
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int32_t t = __shfl_sync(0xffffffffu, tok, (i + j) & 31);
            if (i + j < used && left > 0) v[j].load(dout + (int64_t)t * a.ldo, left);
        }
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int32_t kj = __shfl_sync(0xffffffffu, k, (i + j) & 31), kn = __shfl_sync(0xffffffffu, k, (i + j + 1) & 31);
            if (i + j >= used) continue;
            sum.add(v[j]);
            const bool end = i + j + 1 == len;
            if (!end && kn == kj) continue;
            // a run ends here, or the block does
            if (left > 0) {
                if ((first_run && head) || (end && tail)) sum.put(part + (first_run && head ? 0 : a.d), left);
                else sum.store(static_cast<E *>(a.dtable) + (int64_t)kj * a.d + col, left, a.scale);
            }
            sum.fill(0.0f);
            first_run = false;
        }
    }
}

// Words whose tokens span blocks: the partial sums in order, by the threads of the block where the word begins
template <typename E, int VEC, int STEP> __global__ void __launch_bounds__(256) k_embed_join(const SumArgs a)
{
    griddep_wait();
    griddep_launch_dependents();
    const int64_t b = (int64_t)blockIdx.x * (256 >> a.log_tx) + (threadIdx.x >> a.log_tx);
    const int64_t col = first_col<VEC, STEP>(a.log_tx), left = a.d - col;
    const int64_t blocks = ((int64_t)a.T + kRun - 1) / kRun, p0 = b * kRun;
    if (left <= 0 || b + 1 >= blocks) return;
    const int32_t k = a.keys[p0 + kRun - 1], next = a.keys[p0 + kRun], prev = b > 0 ? a.keys[p0 - 1] : -1;
    if (k >= a.V || next != k || prev == k) return;
    Cols<E, VEC, STEP> sum;
    sum.get(a.part + (b * 2 + 1) * a.d + col, left);
    constexpr int F = 8;
    bool more = true;
    for (int64_t i = b + 1; more && i < blocks; i += F) {   // (a block that has none of the word has no partial sum: loaded, not used)
        Cols<E, VEC, STEP> x[F];
        bool has[F];
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int64_t at = i + j < blocks ? i + j : blocks - 1;
            has[j] = i + j < blocks && a.keys[at * kRun] == k;
            x[j].get(a.part + at * 2 * a.d + col, left);
        }
        asm volatile("" ::: "memory");   // (all of them in flight, not one after the other)
#pragma unroll
        for (int j = 0; j < F; ++j)
            if (has[j]) sum.add(x[j]);
        more = has[F - 1];
    }
    sum.store(static_cast<E *>(a.dtable) + (int64_t)k * a.d + col, left, a.scale);
}

// How threads cover a row: whole vectors, 2^log threads along it (32 at least: a warp's threads share their rows), or four
// single columns a thread, 256 apart, or 32 apart in rows of up to 128
struct Cover {
    int log_tx;
    unsigned cols;   // CTAs along a row
};
template <int V16> Cover cover(int64_t d, bool vec, int least)
{
    Cover c;
    if (!vec) {
        c.log_tx = d <= 128 ? 5 : 8;
        c.cols = (unsigned)((d + (4 << c.log_tx) - 1) >> (c.log_tx + 2));
        return c;
    }
    const int64_t n = d / V16;
    c.log_tx = least;
    while (c.log_tx < 8 && (int64_t(1) << c.log_tx) < n) ++c.log_tx;
    c.cols = (unsigned)((n + (int64_t(1) << c.log_tx) - 1) >> c.log_tx);
    return c;
}

struct EmbedWs {
    int32_t *keys, *vals;
    float *part;
    size_t bytes;
};
EmbedWs carve(void *ws, int64_t T, int64_t d)
{
    WsCarver w(ws);
    EmbedWs e;
    e.keys = w.take<int32_t>(2 * T);
    e.vals = w.take<int32_t>(2 * T);
    e.part = w.take<float>((T + kRun - 1) / kRun * 2 * d);
    e.bytes = w.used;
    return e;
}

resbm_status check(const resbm_embed_desc *desc, const int64_t *ids, const void *table, const void *out, bool table_dense)
{
    if (!desc) return RESBM_ERR_INVALID_ARG;
    const resbm_embed_desc &d = *desc;
    if (d.flags || !isfinite(d.scale)) return RESBM_ERR_INVALID_ARG;
    const resbm_status st = embed_check_shape(d.T, d.V, d.d, d.dtype);
    if (st != RESBM_OK) return st;
    constexpr int64_t limit = INT64_MAX / 64;
    const int64_t es = d.dtype == RESBM_BF16 ? 2 : 4;
    const bool t = d.T > 0;
    auto bad = [&](int64_t rows, int64_t ld) { return rows > 1 && (ld < d.d || !mul_ok(rows, ld) || rows * ld > limit); };
    if ((!table_dense && bad(d.V, d.ldt)) || bad(d.T, d.ldo)) return RESBM_ERR_INVALID_ARG;
    if (!ptr_ok(ids, 8, t) || !ptr_ok(table, es, t || table_dense) || !ptr_ok(out, es, t)) return RESBM_ERR_INVALID_ARG;
    return RESBM_OK;
}

Range rows_of(const void *p, int64_t n, int64_t ld, int64_t d, int64_t es) { return rng(p, n > 0 ? (n - 1) * (n > 1 ? ld : 0) + d : 0, es); }

template <typename E> cudaError_t run_fwd(const resbm_embed_desc &d, const int64_t *ids, const void *table, void *out, const Ctx &c)
{
    constexpr int V16 = 16 / (int)sizeof(E);
    const bool vec = d.d % V16 == 0 && al16(table) && al16(out) && (d.V == 1 || d.ldt % V16 == 0) && (d.T == 1 || d.ldo % V16 == 0);
    const Cover v = cover<V16>(d.d, vec, 0);
    const int64_t rows = 256 >> v.log_tx, ctas = (d.T + rows - 1) / rows;
    const dim3 grid((unsigned)std::min<int64_t>(ctas, std::max<int64_t>(1, 16 * c.sm_count / (int64_t)v.cols)), v.cols);
    auto go = [&](auto kernel) {
        return launch(kernel, grid, dim3(256), 0, c.stream, ids, static_cast<const E *>(table), d.ldt, static_cast<E *>(out), d.ldo, d.T, d.V, d.d, d.scale, v.log_tx);
    };
    return vec ? go(k_embed_fwd<E, V16, 0>) : v.log_tx == 5 ? go(k_embed_fwd<E, 4, 32>) : go(k_embed_fwd<E, 4, 256>);
}

template <typename E> cudaError_t run_bwd(const resbm_embed_desc &d, const int64_t *ids, const void *dout, void *dtable, const EmbedWs &w, const Ctx &c)
{
    // the digits of 0 .. V
    int width = 1;
    while (width < 31 && (int64_t(1) << width) <= d.V) ++width;
    const int passes = (width + 8) / 9, bits = (width + passes - 1) / passes;
    const uint32_t smem = std::max(32768u, 32u * 4u << bits);   // (the zeros: 32 KB)
    static std::atomic<uint8_t> done[kMaxDev];
    cudaError_t e = ensure_smem(k_sort, 32 * 4 * kMaxBins, c.device, done);
    // (the cluster's size is the kernel's own)
    // Zeros: 64 KB a CTA at least, and no more clusters than can be there at once (two in 18 or 20 SMs): the last ones would wait
    // for others to end, and write 158 MB of 1 GB by themselves
    // (T = 65536, V = 250002, d = 1003 in fp32, forward and backward: 307 us with 13 clusters of zeros, 334 with 11, 348 with 15, 379 with 18)
    const int64_t bytes = d.V * d.d * (int64_t)sizeof(E);
    const int64_t clusters = std::max<int64_t>(1, std::min<int64_t>((bytes + kSortCtas * 65536 - 1) / (kSortCtas * 65536), kZeroClusters));
    const unsigned grid = (unsigned)(kSortCtas * (1 + clusters));
    if (e == cudaSuccess) e = launch(k_sort, dim3(grid), dim3(kSortThreads), smem, c.stream, ids, (int)d.T, (int)d.V, d.padding, passes, bits, w.keys, w.vals,
                                     static_cast<uint8_t *>(dtable), bytes);
    if (e != cudaSuccess) return e;
    constexpr int V16 = 16 / (int)sizeof(E);
    const bool vec = d.d % V16 == 0 && al16(dout) && al16(dtable) && (d.T == 1 || d.ldo % V16 == 0);
    const Cover v = cover<V16>(d.d, vec, 5);
    const int64_t per = 256 >> v.log_tx, blocks = (d.T + kRun - 1) / kRun;
    SumArgs a{w.keys + ((passes - 1) & 1) * d.T, w.vals + ((passes - 1) & 1) * d.T, dout, dtable, w.part, d.ldo, d.d, (int)d.T, (int)d.V, v.log_tx, d.scale};
    const dim3 ctas((unsigned)((blocks + per - 1) / per), v.cols);
    auto go = [&](auto sum, auto join) {
        cudaError_t e = launch(sum, ctas, dim3(256), 0, c.stream, a);
        if (e == cudaSuccess && blocks > 1) e = launch(join, ctas, dim3(256), 0, c.stream, a);
        return e;
    };
    e = vec ? go(k_embed_sum<E, V16, 0>, k_embed_join<E, V16, 0>)
        : v.log_tx == 5 ? go(k_embed_sum<E, 4, 32>, k_embed_join<E, 4, 32>) : go(k_embed_sum<E, 4, 256>, k_embed_join<E, 4, 256>);
    if (e == cudaSuccess) count_launches(blocks > 1 ? 3 : 2);
    return e;
}

}  // namespace

resbm_status embed_check_shape(int64_t T, int64_t V, int64_t d, int32_t dtype)
{
    if (T < 0 || V < 1 || d < 1 || (dtype != RESBM_F32 && dtype != RESBM_BF16)) return RESBM_ERR_INVALID_ARG;
    constexpr int64_t most = int64_t(1) << 29;
    return T >= most || V >= most || d > (int64_t(1) << 20) ? RESBM_ERR_UNSUPPORTED : RESBM_OK;
}

size_t embed_bwd_ws_bytes(int64_t T, int64_t d) { return carve(nullptr, T, d).bytes; }

}  // namespace resbm

using namespace resbm;

extern "C" {

resbm_status resbm_embed_fwd(const resbm_embed_desc *desc, const int64_t *ids, const void *table, void *out, void *stream)
{
    resbm_status st = check(desc, ids, table, out, false);
    if (st != RESBM_OK) return st;
    const resbm_embed_desc &d = *desc;
    const int64_t es = d.dtype == RESBM_BF16 ? 2 : 4;
    const Range o = rows_of(out, d.T, d.ldo, d.d, es);
    if (overlaps(o, rows_of(table, d.V, d.ldt, d.d, es)) || overlaps(o, rng(ids, d.T, 8))) return RESBM_ERR_INVALID_ARG;
    Ctx c;
    st = make_ctx(stream, &c);
    if (st != RESBM_OK || d.T == 0) return st;
    const cudaError_t e = d.dtype == RESBM_F32 ? run_fwd<float>(d, ids, table, out, c) : run_fwd<__nv_bfloat16>(d, ids, table, out, c);
    if (e == cudaSuccess) count_launches(1);
    else cudaGetLastError();
    return finish(e);
}

resbm_status resbm_embed_bwd(const resbm_embed_desc *desc, const int64_t *ids, const void *dout, void *dtable, void *ws, size_t ws_bytes, void *stream)
{
    resbm_status st = check(desc, ids, dtable, dout, true);
    if (st != RESBM_OK) return st;
    const resbm_embed_desc &d = *desc;
    const int64_t es = d.dtype == RESBM_BF16 ? 2 : 4;
    if (!ptr_ok(ws, 256, false)) return RESBM_ERR_INVALID_ARG;
    const Range outs[] = {rng(dtable, d.V * d.d, es), rng(ws, (int64_t)std::min<size_t>(ws_bytes, INT64_MAX), 1)};
    const Range ins[] = {rows_of(dout, d.T, d.ldo, d.d, es), rng(ids, d.T, 8)};
    if (any_overlap(outs, ins, 2)) return RESBM_ERR_INVALID_ARG;
    if (d.T > 0 && (!ws || ws_bytes < embed_bwd_ws_bytes(d.T, d.d))) return RESBM_ERR_WORKSPACE;
    Ctx c;
    st = make_ctx(stream, &c);
    if (st != RESBM_OK) return st;
    if (d.T == 0) return finish(cudaMemsetAsync(dtable, 0, (size_t)(d.V * d.d * es), c.stream));
    const EmbedWs w = carve(ws, d.T, d.d);
    const cudaError_t e = d.dtype == RESBM_F32 ? run_bwd<float>(d, ids, dout, dtable, w, c) : run_bwd<__nv_bfloat16>(d, ids, dout, dtable, w, c);
    if (e != cudaSuccess) cudaGetLastError();
    return finish(e);
}

}  // extern "C"
