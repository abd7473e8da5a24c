// vocab_gemm.cuh -- the four products of the vocabulary's losses (include/resbm_vocab.h) on tcgen05, each with the step
// that follows it applied to the accumulator before it leaves the chip.
//
//   VG_FWD   z = X . W^T             a row's running maximum and sum of exponentials over the unit's columns, and its
//                                    targets' logits: 16 bytes a row and unit instead of the logits
//   VG_DZ    z again, then           dz = g (softmax(z / tau) - q), stored for a piece of the vocabulary at a time (bf16: over the g's
//                                    common factor, whose rounding would be the same for every token's label)
//   VG_DX    dz . W                  fp32, added to what earlier pieces gave
//   VG_DW    dz^T . X                complete for the piece's rows of W (in one launch with VG_DX)
//
// X: the n tokens that have a target, packed (n is on the device only); z and dz have a row for each of them.
//
// Work units are (256 rows, up to 256 columns, depth split), unit u on CTA pair u mod pairs, row blocks in groups of
// `group` with the columns outside, so that the pairs at work share operands in L2. A pair (cta_group::2) has per CTA
//   producer warp  : TMA loads of 64-deep slices of its 128 rows of A and its half of B, 128-byte swizzle, six stages
//   MMA warp       : (even CTA) four 256 x bn x 16 products a slice into one of two TMEM accumulators
//   epilogue warps : eight, two a TMEM lane quarter with half of the columns each, one row a thread
// and the next unit's products overlap this unit's epilogue.
//
// fp32 (SPLIT 3): every operand is the sum of three bf16 values (the value rounded, its remainder rounded, and once more:
// 24 bits), and a product the six of nine partial ones that are over 2^-24 of it, smallest first. They are one product of
// six times the depth at the bf16 rate: 320 TFLOP/s of fp32 at most, where CUDA cores have 75.
//
// Few tokens in use in bf16 (SPLIT 2, up to kTwoParts of them): dz as two bf16 values. Its rounding is one of the outputs' own size, but a
// single token's gradients have one large dz, the label's, whose error no sum averages: up to 2^-8 of the whole of dX and dW (T = 1:
// 3.7e-3 off). Over more tokens dW averages them, and dX's norm its rows: 2.3e-3 of it instead of 1.7e-3. (One token, V = 32000, d = 2048,
// forward and backward: 144 us with one part, 165 with two.) How many are in use is known on the device, so one kernel has both forms;
// the second part of the 64 rows that a slice of dW's depth reads lies kRest rows on, in the same row block.
//
// PIECES: the tensor core truncates as it adds to its accumulator, an error that grows with the number of MMAs in one
// accumulator (run_loss has figures). Where that is seen in an output (the logits, and everything in fp32) a unit's sum
// runs in pieces, which alternate between the accumulators; the epilogue warps add them in registers, rounded to
// nearest, while the next piece runs.
//
// What bounds it: with d of 2048 and more the tensor cores (T = 2048, V = 32000, d = 2048: 144 us forward, 157 dz, 283 both
// gradients, 1710 to 1900 TFLOP/s; in a long run the board's power, 1.7 PFLOP/s); with d under 512 the epilogue, whose
// warps wait for their own results most of the time (T = 8192, V = 32000, d = 128 130 us forward, where the tensor cores need 38 and
// the exponentials 57). Sixteen epilogue warps of 64 columns took 235: what a unit costs a warp apart from its columns, and 96
// registers a thread, which spill. The logits' targets are looked up by bisection in a token's sorted list, and a label is a
// list of one.
//
// Every element is summed by one CTA in a fixed order, and a depth split has a slot of its own: results are the same bits
// every time.
#pragma once

#include <limits.h>
#include <math.h>

#include "common.cuh"
#include "pair.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace resbm {
namespace tc {

enum VocabMode : int { VG_FWD, VG_DZ, VG_DX, VG_DW, VG_GRADS };   // GRADS: units of DX and of DW in one launch

struct VocabGemm {
    int32_t mode;             // of VG_GRADS: VG_DX or VG_DW
    const int32_t *n_ptr;     // tokens in use: *n_ptr, or n_rows where it is null
    int32_t n_rows;
    int32_t rows;             // VG_DW: rows of the piece (words)
    int32_t cols;             // columns that exist
    int32_t depth;            // FWD, DZ, DX
    int32_t bn, nn;           // columns a unit (a multiple of 32), units along the columns
    int32_t splits, group;
    int32_t a_off, b_off;     // rows from one of three parts of an operand to the next
    int32_t a_rows;           // FWD, DZ, DX: rows of A a load: 128, or fewer where one load has all tokens
    int32_t b_y;              // FWD, DZ, DX: the piece's first row in B's tensor map
    int32_t out_y;            // DW: the piece's first row of dW
    int32_t slot_rows;        // DX, DW: rows of a slot
    int32_t add;              // DX: added to the slots
    // the rows' tokens, targets and scalars (FWD, DZ)
    int32_t v0;               // the piece's first word
    const int32_t *token;     // row -> token, or null: the same
    const int64_t *label;     // a token's target, or null: the lists
    const int2 *list;         // K targets a token in ascending order with their weights' bits, INT32_MAX behind the last
    int32_t K;
    int32_t slot0;            // FWD: the first slot of this launch (two a unit)
    int64_t tp;               // rows of a slot, rounded up
    float c;                  // log2(e) / tau
    float2 *stat;             // FWD: (maximum c, sum of 2^(z c - maximum c)) of slot, row
    float *zt;                // FWD: the label's logit a row; with lists: the weighted sum of slot, row
    const float *lse, *dloss; // DZ: a token's log-sum-exp, its loss's gradient
    const float *scale;       // bf16: the losses' gradients' common factor, and that times tau; dz is without it, the gradients get it at the end
    int32_t dloss_step;       // 1, or 0: one for all
    float tau;
    const float *bad;         // DZ: a value added to a token's gradient (NaN where its targets are none), or null
    int32_t V;
    // DW where TMA cannot store: the matrix, its pitch in elements
    void *out;
    int64_t ldo;
    int32_t out_f32;          // DW: fp32 result (slots, or an fp32 dW), else bf16
};

constexpr int kTwoParts = 16, kRest = 128;

struct VocabCfg {
    static constexpr uint32_t A_STAGE = 128 * 128, B_STAGE = 128 * 128, STAGE = A_STAGE + B_STAGE;
    static constexpr int NST = 6;
    static constexpr uint32_t BOX = 4096;                   // staging of an epilogue warp: 32 rows of 32 fp32, or two of bf16
    static constexpr uint32_t OFF_BOX = NST * STAGE;
    static constexpr uint32_t SMEM = OFF_BOX + 8 * BOX + 1024;
    static_assert(SMEM <= 232448 - 512, "shared memory budget");
    static constexpr int THREADS = 320;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// add a box to global memory (fp32), element by element
__device__ __forceinline__ void tma_add_2d(const CUtensorMap *m, int32_t x, int32_t y, uint32_t src)
{
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                     reinterpret_cast<uint64_t>(m)),
                 "r"(x), "r"(y), "r"(src)
                 : "memory");
}

// A row's targets in ascending order, seen from a tile: `next` is the next one's column in the tile (INT_MAX: none).
struct Targets {
    const int2 *list;
    int K, p, base, next;
    float q;
    __device__ __forceinline__ void set()
    {
        next = INT_MAX;
        if (p < K) {
            const int2 v = list[p];
            if (v.x != INT32_MAX) {
                next = v.x - base;
                q = __int_as_float(v.y);
            }
        }
    }
    // those from column `first` of the tile that starts at word `base_` on
    __device__ __forceinline__ void start(const VocabGemm &g, int64_t token, int32_t label, int base_, int first)
    {
        base = base_;
        if (g.label) {
            K = 0;
            q = 1.0f;
            next = label >= base + first && label != INT32_MAX ? label - base : INT_MAX;
            return;
        }
        K = g.K;
        list = g.list + token * K;
        int lo = 0, hi = K;   // the first with list >= base + first
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (list[mid].x < base + first) lo = mid + 1;
            else hi = mid;
        }
        p = lo;
        set();
    }
    __device__ __forceinline__ void advance()
    {
        if (K == 0) {
            next = INT_MAX;
        } else {
            ++p;
            set();
        }
    }
};

// What a row's token brings along, loaded a unit ahead (three loads that wait for one another, 1500 cycles)
struct RowIn {
    int32_t token, label;
    float lse, dloss, bad;
};

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// x / d for x under 2^31: a product with the reciprocal and a correction (a division is 20 dependent instructions, and every warp
// has three a unit)
struct Divisor {
    uint32_t d, m;
    __device__ __forceinline__ void set(uint32_t d_)
    {
        d = d_ ? d_ : 1;
        m = 0xFFFFFFFFu / d;   // (2^32 / d or up to one less: a quotient is right or one less)
    }
    __device__ __forceinline__ uint32_t of(uint32_t x) const
    {
        const uint32_t q = __umulhi(x, m);
        return q + (x - q * d >= d);
    }
};

// JOBS: 1, or the two of VG_GRADS, whose units follow one another (the one with the longer units first): apart, the last round of
// each leaves pairs without work.
template <int JOBS> struct VocabJobs {
    CUtensorMap a[JOBS], b[JOBS], o[JOBS];
    VocabGemm g[JOBS];
};

// MODE: what becomes of the accumulator; SPLIT: bf16 parts of an operand (2: of dz alone, for few tokens); PIECE: 64-deep slices of a piece of a
// sum (0: whole)
template <int MODE, int SPLIT, int PIECE, int JOBS>
__global__ void __launch_bounds__(VocabCfg::THREADS, 1) k_vocab_gemm(const __grid_constant__ VocabJobs<JOBS> jobs)
{
    using C = VocabCfg;
    constexpr bool GRADS = MODE == VG_GRADS, BMN = GRADS;
    constexpr bool PIECES = PIECE > 0;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[C::NST], empty[C::NST], acc_full[2], acc_empty[2], done_bar;
    __shared__ uint32_t tmem_base_sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t crank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::NST; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&acc_full[i]), 1);
            mbar_init(smem_u32(&acc_empty[i]), 16);   // both CTAs' epilogue warps, on the even CTA
        }
        mbar_init(smem_u32(&done_bar), 1);
        fence_mbar_init();
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_base_sh), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    griddep_wait();
    griddep_launch_dependents();
    const uint32_t tmem = tmem_base_sh;

    // the units, in every warp alike
    const int n = jobs.g[0].n_ptr ? *jobs.g[0].n_ptr : jobs.g[0].n_rows;
    const bool two = SPLIT == 2 && n <= kTwoParts;   // dz in two parts
    const int terms = SPLIT == 3 ? 6 : GRADS && two ? 2 : 1;
    struct Job {
        bool dw;
        int rows, slices, per;
        uint32_t nm, per_split, units;
        Divisor split, group, rows_left, whole;   // units a split, a group of row blocks; row blocks of the last group, of the others
    };
    const uint32_t group = (uint32_t)jobs.g[0].group;
    auto job_of = [&](int j) {
        const VocabGemm &g = jobs.g[j];
        Job k;
        k.dw = GRADS && g.mode == VG_DW;
        k.rows = k.dw ? g.rows : n;
        k.slices = ((k.dw ? n : g.depth) + 63) / 64;
        k.per = (k.slices + g.splits - 1) / g.splits;
        k.nm = (uint32_t)((k.rows + 255) / 256);
        k.per_split = k.nm * (uint32_t)g.nn;
        k.units = k.per_split * (uint32_t)g.splits;
        if (GRADS) k.split.set(k.per_split);
        k.group.set(group * (uint32_t)g.nn);
        k.rows_left.set(k.nm % group);
        k.whole.set(group);
        return k;
    };
    const Job job0 = job_of(0), job1 = job_of(JOBS - 1);
    const uint32_t units = job0.units + (JOBS > 1 ? job1.units : 0);
    // This pair's i-th unit. One job: every pairs-th one. Two: the pairs that got one unit of the first job fewer take `extra` of the
    // second one's, about as much work, before all of them go on in turn. (In plain turns 104 units of 256 slices and then 504 of
    // 52 leave some pairs 876 slices where the mean is 695; so 724.)
    constexpr uint32_t kUnitSlices = 6;   // what a unit costs around its products
    const uint32_t pair = cluster_index(), pairs = gridDim.x / 2;
    const uint32_t mine0 = pair < job0.units ? (job0.units - pair + pairs - 1) / pairs : 0;
    const int over = JOBS > 1 ? (int)(job0.units % pairs) : 0;
    const uint32_t under = pairs - over;
    const bool late = (int)pair >= over;
    uint32_t extra = 0;
    if (JOBS > 1 && over > 0) {
        const uint32_t c0 = (uint32_t)terms * job0.per + kUnitSlices, c1 = (uint32_t)terms * job1.per + kUnitSlices;
        extra = (2 * c0 + c1) / (2 * c1);
        if (extra > job1.units / under) extra = job1.units / under;
    }
    auto unit_at = [&](uint32_t i) -> uint32_t {
        if (i < mine0) return pair + i * pairs;
        if (JOBS == 1) return units;
        i -= mine0;
        uint32_t t;
        if (late && i < extra) t = i * under + pair - over;
        else t = extra * under + pair + (i - (late ? extra : 0)) * pairs;
        return job0.units + t;   // (units or more: none)
    };
    // a unit: its job, 128-row block of this CTA, column block, split, slices [k0, k0 + nk)
    struct Unit {
        int job, mb, nb, ks, k0, nk;
    };
    auto unit_of = [&](uint32_t u) {
        Unit x;
        auto decode = [&](const Job &k, uint32_t r) {
            x.ks = 0;
            if (GRADS) {   // (the others are not split)
                x.ks = (int)k.split.of(r);
                r -= (uint32_t)x.ks * k.per_split;
            }
            const uint32_t gi = k.group.of(r);
            r -= gi * k.group.d;
            const bool last = k.nm - gi * group < group;
            x.nb = (int)(last ? k.rows_left.of(r) : k.whole.of(r));
            x.mb = 2 * (int)(gi * group + r - (uint32_t)x.nb * (last ? k.rows_left.d : group)) + (int)crank;
            x.k0 = x.ks * k.per;
            const int k1 = x.k0 + k.per < k.slices ? x.k0 + k.per : k.slices;
            x.nk = k1 > x.k0 ? k1 - x.k0 : 0;
        };
        x.job = JOBS > 1 && u >= job0.units;
        if (x.job) decode(job1, u - job0.units);
        else decode(job0, u);
        return x;
    };

    if (warp == 0) {
        // ---------------- producer ----------------
        if (elect_one()) {
            for (int j = 0; j < JOBS; ++j) {
                tma_prefetch_desc(&jobs.a[j]);
                tma_prefetch_desc(&jobs.b[j]);
            }
            uint32_t it = 0;
            bool ok = true;
            for (uint32_t i = 0, u; (u = unit_at(i)) < units && ok; ++i) {
                const Unit x = unit_of(u);
                const VocabGemm &g = jobs.g[x.job];
                const CUtensorMap *ma = &jobs.a[x.job], *mb = &jobs.b[x.job];
                const bool dw = GRADS && (x.job ? job1.dw : job0.dw);
                const int half_b = g.bn / 2;   // this CTA's columns of B
                const int loads_b = BMN ? (half_b + 63) / 64 : 1;
                // Few tokens: the rows of A behind them are not loaded (rows that the tensor map fills cost more than rows that it
                // reads: T = 1 took 47 us where T = 32 took 32), and what stands there goes into rows of the product that nobody reads.
                const bool few = !dw && g.a_rows < 128;
                const uint32_t bytes_a = few ? (uint32_t)g.a_rows * 128u : 2 * C::A_STAGE;
                const uint32_t bytes = bytes_a + 2 * (BMN ? (uint32_t)loads_b * 8192u : (uint32_t)half_b * 128u);
                const int row = x.mb * 128, col = x.nb * g.bn + (int)crank * half_b;
                const int piece = PIECES ? PIECE : x.nk;
                for (int kp = 0; kp < x.nk && ok; kp += piece) {
                    const int ke = x.nk - kp < piece ? x.nk : kp + piece;
                    // a slice of the operands' parts whose rows begin ya and yb on
                    auto load = [&](int ya, int yb, int k) {
                        const uint32_t s = it % C::NST, ph = (it / C::NST) & 1, own = smem_u32(&full[s]), bar = map_shared(own, 0);
                        const uint32_t ad = smem_u32(smem + s * C::STAGE), bd = ad + C::A_STAGE;
                        if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1)) {
                            ok = false;
                            return;
                        }
                        if (crank == 0) mbar_expect_tx(own, bytes);   // both CTAs' bytes
                        if (!dw) {
                            if (!few || crank == 0) tma_load_2d_pair(ad, ma, k, ya + row, bar);
                        } else {
                            tma_load_2d_pair(ad, ma, row, ya + k, bar);
                            tma_load_2d_pair(ad + 8192, ma, row + 64, ya + k, bar);
                        }
                        if (!BMN) {
                            tma_load_2d_pair(bd, mb, k, yb + col, bar);
                        } else {   // (what lies past the half is loaded and not read)
                            for (int j = 0; j < loads_b; ++j) tma_load_2d_pair(bd + j * 8192, mb, col + 64 * j, yb + k, bar);
                        }
                        ++it;
                    };
                    const int first = 64 * (x.k0 + kp), end = 64 * (x.k0 + ke);
                    if constexpr (SPLIT == 2 && GRADS) {   // dz's remainder, dz; slice by slice: the second product finds W's in L2
                        for (int k = first; k < end && ok; k += 64) {
                            if (two) load(kRest, g.b_y, k);
                            if (ok) load(0, g.b_y, k);
                        }
                    } else {
#pragma unroll 1
                        for (int term = 0; term < terms && ok; ++term) {
                            // the partial products, smallest first: (2, 0) (1, 1) (0, 2) (1, 0) (0, 1) (0, 0)
                            const int sa = SPLIT < 3 ? 0 : term == 0 ? 2 : (term == 1 || term == 3) ? 1 : 0;
                            const int sb = SPLIT < 3 ? 0 : term == 2 ? 2 : (term == 1 || term == 4) ? 1 : 0;
                            const int ya = sa * g.a_off, yb = sb * g.b_off + g.b_y;
                            for (int k = first; k < end && ok; k += 64) load(ya, yb, k);
                        }
                    }
                }
            }
            // the MMAs that read the last stages have completed before the CTA may leave
            const uint32_t last = it < (uint32_t)C::NST ? it : (uint32_t)C::NST;
            for (uint32_t i = 0; i < last && ok; ++i) {
                const uint32_t j = it - 1 - i;
                mbar_wait(smem_u32(&empty[j % C::NST]), (j / C::NST) & 1);
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (crank == 0 && elect_one()) {
            const uint32_t a0 = smem_u32(smem), b0 = a0 + C::A_STAGE;
            const uint64_t bd0 = BMN ? smem_desc(b0, 8192, 1024, kSwz128) : smem_desc(b0, 16, 1024, kSwz128);
            constexpr uint64_t BK = (BMN ? 2048 : 32) >> 4;
            uint32_t it = 0, ti = 0;
            bool ok = true;
            for (uint32_t i = 0, u; (u = unit_at(i)) < units && ok; ++i) {
                const Unit x = unit_of(u);
                const bool dw = GRADS && (x.job ? job1.dw : job0.dw);   // A: dz^T, a row of it along the lines of memory
                const uint32_t idesc = idesc_bf16(256, (uint32_t)jobs.g[x.job].bn, dw, BMN);
                const uint64_t ad0 = dw ? smem_desc(a0, 8192, 1024, kSwz128) : smem_desc(a0, 16, 1024, kSwz128);
                const uint64_t AK = (dw ? 2048 : 32) >> 4;
                const int piece = PIECES ? PIECE : x.nk;
                for (int kp = 0; kp < x.nk && ok; kp += piece) {
                    const uint32_t ab = ti & 1;
                    ok = mbar_wait(smem_u32(&acc_empty[ab]), ((ti >> 1) & 1) ^ 1);
                    tc_fence_after();
                    if (!ok) break;
                    const int steps = (x.nk - kp < piece ? x.nk - kp : piece) * terms;
                    for (int i = 0; i < steps; ++i, ++it) {
                        const uint32_t s = it % C::NST, ph = (it / C::NST) & 1;
                        ok = mbar_wait(smem_u32(&full[s]), ph);
                        tc_fence_after();
                        if (!ok) break;
                        const uint64_t so = (uint64_t)((s * C::STAGE) >> 4);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_bf16_pair(tmem + ab * 256, ad0 + so + kk * AK, bd0 + so + kk * BK, idesc, i > 0 || kk > 0);
                        mma_commit_pair(smem_u32(&empty[s]));
                    }
                    if (!ok) break;
                    mma_commit_pair(smem_u32(&acc_full[ab]));
                    ++ti;
                }
            }
            mma_commit_pair(smem_u32(&done_bar), 1);
            mbar_wait(smem_u32(&done_bar), 0);
        }
    } else {
        // ---------------- epilogue warps ----------------
        const int q = warp & 3, half = (warp - 2) >> 2;   // TMEM lane quarter, which half of the columns
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        uint8_t *const box = smem + C::OFF_BOX + (warp - 2) * C::BOX;
        uint32_t ti = 0, boxes = 0;
        bool ok = true, whole_box = false;   // the last store came from the whole box (fp32), not from a half of it

        auto release_acc = [&](uint32_t ab) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(map_shared(smem_u32(&acc_empty[ab]), 0));
        };
        // 32 columns of this thread's row as bf16: the next of the two 2 KB boxes, stored at (col, row0)
        auto store_bf16 = [&](const CUtensorMap *mo, const float (&v)[32], int col, int row0) {
            // (VG_GRADS: a unit of DX before this one of DW may still have its 4 KB read)
            if (lane == 0) {
                if (GRADS && whole_box) bulk_wait_read<0>();
                else bulk_wait_read<1>();
            }
            whole_box = false;
            __syncwarp();
            uint8_t *b = box + (boxes++ & 1) * 2048;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<uint4 *>(b + swz_offset((uint32_t)lane, 16 * e, 64)) =
                    make_uint4(pack_bf16(v[8 * e], v[8 * e + 1]), pack_bf16(v[8 * e + 2], v[8 * e + 3]),
                               pack_bf16(v[8 * e + 4], v[8 * e + 5]), pack_bf16(v[8 * e + 6], v[8 * e + 7]));
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                tma_store_2d(mo, col, row0, smem_u32(b));
                bulk_commit();
            }
        };
        auto store_f32 = [&](const CUtensorMap *mo, const float (&v)[32], int col, int row0, bool add) {
            if (lane == 0) bulk_wait_read<0>();
            whole_box = true;
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                *reinterpret_cast<float4 *>(box + swz_offset((uint32_t)lane, 16 * e, 128)) =
                    make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (add) tma_add_2d(mo, col, row0, smem_u32(box));
                else tma_store_2d(mo, col, row0, smem_u32(box));
                bulk_commit();
            }
        };
        // DW into a matrix off the 16-byte grid: a row at a time, one element a lane
        auto store_plain = [&](const VocabGemm &g, const float (&v)[32], int col, int row0) {
            if (lane == 0) bulk_wait_read<0>();   // (a unit of DX before this one)
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                *reinterpret_cast<float4 *>(box + swz_offset((uint32_t)lane, 16 * e, 128)) =
                    make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            __syncwarp();
            if (col + lane < g.cols) {
                for (int r = 0; r < 32 && row0 + r < g.rows; ++r) {
                    const float x = *reinterpret_cast<const float *>(box + swz_offset((uint32_t)r, 4 * lane, 128));
                    const int64_t at = (int64_t)(g.out_y + row0 + r) * g.ldo + col + lane;
                    if (g.out_f32) static_cast<float *>(g.out)[at] = x;
                    else static_cast<__nv_bfloat16 *>(g.out)[at] = __float2bfloat16_rn(x);
                }
            }
        };

        auto row_in = [&](const Unit &x) {
            RowIn r = {};
            if (GRADS) return r;
            const VocabGemm &g = jobs.g[0];
            const int row = x.mb * 128 + q * 32 + lane;
            if (row >= n) return r;
            r.token = g.token ? g.token[row] : row;
            if (g.label) {
                const int64_t y = g.label[r.token];
                r.label = y < 0 ? -1 : y < g.V ? (int32_t)y : INT32_MAX;
            }
            if (MODE == VG_DZ) {
                r.lse = g.lse[r.token];
                // (one for all is the factor itself)
                if (SPLIT == 2) r.dloss = g.dloss_step ? g.dloss[r.token] / g.scale[0] : 1.0f;
                else r.dloss = g.dloss[(int64_t)r.token * g.dloss_step] * g.tau;
                if (g.bad) r.bad = g.bad[r.token];
            }
            return r;
        };
        const float factor = SPLIT == 2 && GRADS ? jobs.g[0].scale[1] : 1.0f;   // (of slots: k_finish)
        const float inv_tau = SPLIT == 3 && MODE == VG_DZ ? 1.0f / jobs.g[0].tau : 1.0f;
        uint32_t u = unit_at(0);
        Unit ahead = {};
        if (u < units) ahead = unit_of(u);
        RowIn coming = row_in(ahead);
        for (uint32_t turn = 1; u < units && ok; ++turn) {
            const Unit x = ahead;
            const VocabGemm &g = jobs.g[x.job];
            const CUtensorMap *mo = &jobs.o[x.job];
            const bool dw = GRADS && (x.job ? job1.dw : job0.dw);
            const int rows = x.job ? job1.rows : job0.rows;
            const int nb = x.nb, ks = x.ks, nk = x.nk;
            const int groups = g.bn / 32, first_group = half ? (groups + 1) / 2 : 0;
            const int my = half ? groups / 2 : (groups + 1) / 2;   // groups of 32 columns, up to 4
            const int row0 = x.mb * 128 + q * 32, row = row0 + lane;
            const RowIn in = coming;
            u = unit_at(turn);
            if (u < units) {
                ahead = unit_of(u);
                coming = row_in(ahead);
            }
            // this thread's row
            Targets t;
            t.next = INT_MAX;
            t.K = 0;
            float most = -INFINITY, sum_e = 0.0f, zt = 0.0f, lse2 = 0.0f, grad = 0.0f;
            bool hit = false;
            if (!GRADS && row < n) {
                t.start(g, in.token, in.label, g.v0 + nb * g.bn, first_group * 32);
                if (MODE == VG_DZ) {
                    lse2 = SPLIT == 3 ? in.lse : in.lse * 1.4426950408889634f;
                    grad = in.dloss + in.bad;
                    if (g.label && in.label == INT32_MAX) grad = NAN;
                }
            }
            // what becomes of 32 columns of the row, from column `c` of the tile on
            auto process = [&](float (&v)[32], int c) {
                const int col = nb * g.bn + c;
                if (MODE == VG_DZ) {
                    if (col >= g.cols) return;
                    if (row < n) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            // (fp32: lse times log2(e) has a rounding of its own, the same for the whole row)
                            if (SPLIT == 3) v[j] = exp2_fast(fmaf(v[j], inv_tau, -lse2) * 1.4426950408889634f);
                            else v[j] = exp2_fast(fmaf(v[j], g.c, -lse2));
                        }
                        while (t.next < c + 32) {
                            const int at = t.next - c;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j == at) v[j] -= t.q;
                            t.advance();
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= grad;
                    } else {   // zeros up to the end of the row block: VG_DW's depth ends inside it
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                    }
                    if (two && row0 >= 64) return;
#pragma unroll
                    for (int part = 0; part < SPLIT; ++part) {
                        store_bf16(mo, v, col, part * (SPLIT == 2 ? kRest : g.slot_rows) + row0);
                        if (SPLIT == 2 && !two) break;
                        if (part + 1 < SPLIT) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
                        }
                    }
                } else {
                    if (row0 >= rows || col >= g.cols) return;
                    if (SPLIT == 2 && dw && !g.out_f32) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= factor;
                    }
                    if (!dw) store_f32(mo, v, col, ks * g.slot_rows + row0, g.add);
                    else if (g.out) store_plain(g, v, col, row0);
                    else if (g.out_f32) store_f32(mo, v, col, g.out_y + ks * g.slot_rows + row0, false);
                    else store_bf16(mo, v, col, g.out_y + row0);
                }
            };
            if (nk == 0) {   // nothing to add up: zeros (no token in use, or a split past the end)
                if (GRADS) {
#pragma unroll 1
                    for (int i = 0; i < my; ++i) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                        process(v, (first_group + i) * 32);
                    }
                }
                continue;
            }
            if constexpr (PIECES) {
                float sum[4][32];   // this row's columns
                // a piece's sums out of the accumulator (16 columns at a time: 32 spill)
                auto drain = [&](auto first) {
                    const uint32_t ab = ti & 1;
                    ok = mbar_wait(smem_u32(&acc_full[ab]), (ti >> 1) & 1);
                    tc_fence_after();
                    if (!ok) return;
                    if (row0 < rows) {   // (the same for the whole warp)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (i < my) {
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float v[16];
                                    tmem_ld16(tmem + lane_base + ab * 256 + (first_group + i) * 32 + 16 * h, v);
                                    tmem_ld_wait();
                                    tmem_regs_ready(v);
#pragma unroll
                                    for (int j = 0; j < 16; ++j) sum[i][16 * h + j] = decltype(first)::value ? v[j] : sum[i][16 * h + j] + v[j];
                                }
                            }
                        }
                    }
                    release_acc(ab);
                    ++ti;
                };
                int kp = 0;
                if constexpr (MODE == VG_FWD) {   // (the others spill with it)
                    drain(Yes());
                    kp = PIECE;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[i][j] = 0.0f;
                }
#pragma unroll 1
                for (; kp < nk && ok; kp += PIECE) drain(No());
                if (!ok) break;
                if constexpr (MODE == VG_FWD) {
                    if (row < n) {
                        // the targets' logits, then the maximum and the sum of exponentials over what columns exist
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int c = (first_group + i) * 32, left = i < my ? g.cols - nb * g.bn - c : 0;
                            if (left < 32) {
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (j >= left) sum[i][j] = -INFINITY;
                            }
                            // (only in columns that exist: past a piece's end stand the next one's words)
                            while (i < my && t.next < c + min(left, 32)) {
                                const int at = t.next - c;
                                float x = 0.0f;
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (j == at) x = sum[i][j];
                                zt = fmaf(t.q, x, zt);
                                hit = true;
                                t.advance();
                            }
                        }
                        float m[8], s[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) m[j] = sum[0][j];
#pragma unroll
                        for (int j = 8; j < 128; ++j) m[j & 7] = max_nan(m[j & 7], sum[j >> 5][j & 31]);
#pragma unroll
                        for (int w = 4; w; w >>= 1)
#pragma unroll
                            for (int j = 0; j < w; ++j) m[j] = max_nan(m[j], m[j + w]);
                        most = m[0] * g.c;
                        if (!(most == -INFINITY)) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) s[j] = exp2_fast(fmaf(sum[0][j], g.c, -most));
#pragma unroll
                            for (int j = 8; j < 128; ++j) s[j & 7] += exp2_fast(fmaf(sum[j >> 5][j & 31], g.c, -most));
                            sum_e = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
                        }
                        const int64_t at = (int64_t)(g.slot0 + 2 * nb + half) * g.tp + row;   // (of a half without columns too)
                        g.stat[at] = make_float2(most, sum_e);
                        if (!g.label) g.zt[at] = zt;
                        else if (hit) g.zt[row] = zt;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < my) process(sum[i], (first_group + i) * 32);
                }
            } else {
                const uint32_t ab = ti & 1;
                ok = mbar_wait(smem_u32(&acc_full[ab]), (ti >> 1) & 1);
                tc_fence_after();
                if (!ok) break;
#pragma unroll 1
                for (int i = 0; i < my; ++i) {
                    float v[32];
                    tmem_ld32(tmem + lane_base + ab * 256 + (first_group + i) * 32, v);
                    tmem_ld_wait();
                    tmem_regs_ready(v);
                    if (i == my - 1) release_acc(ab);
                    process(v, (first_group + i) * 32);
                }
                if (my == 0) release_acc(ab);
                ++ti;
            }
        }
    }
    if (MODE != VG_FWD && warp >= 2 && lane == 0) bulk_wait<0>();   // this warp's stores are done
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // neither CTA leaves, or frees TMEM, while the other may still address it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

}  // namespace tc
}  // namespace resbm
