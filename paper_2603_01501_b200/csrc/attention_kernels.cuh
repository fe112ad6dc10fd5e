// Device code of causal attention over packed sequences for sm_100a.  Included by attention.cu only.
#pragma once

#include <math.h>
#include <stdint.h>

#include "gac.h"
#include "sm100.cuh"

namespace {

constexpr int kTile = 128;                  // rows of a query or key tile: one tcgen05 accumulator
constexpr float kLog2e = 1.4426950408889634f;

// CTAs so far in which a bounded wait ran out; read by gac_attn_check, never cleared.
static __device__ unsigned g_attn_faults;

struct RowsOut {
    char *p;
    long long token, head;   // bytes
};
struct AttnDev {
    const int32_t *cu;
    uint32_t n_tokens, n_seqs, q_heads, kv_heads, head_dim;
    int q_mul, k_mul, v_mul, do_mul;   // 0 where one head's memory serves all heads (head stride 0), else 1
    float scale, exp2_scale;           // exp2_scale = |scale| log2(e); a negative scale negates q in the product
    uint32_t negate;
    RowsOut o, d_q, d_k, d_v;
    const char *do_in;                 // backward: for the row terms
    long long do_token, do_head;
    float *lse;
    float2 *rows;                      // backward: (-log2(e) lse, row term) of every query head and token
    uint32_t parts;                    // backward: query heads of a group are summed in this many parts,
    uint32_t wait_limit;               // of every wait inside a kernel, in units of 1024 ns
    float *part_sums;                  // kept as binary32 [parts][d_k, d_v][n_tokens][kv_heads][head_dim] when parts > 1
};

// cu_seqlens entry b, kept in range; entry 0 is taken as 0.  The sequences are what a bisection over the entries makes of them:
// the node of entry `mid` cuts its range of tokens at that entry, kept within the range.  Ascending entries are found as
// they are; of entries out of order those nearer the root count, and the sequences still lie one behind the other, which
// is what gives every row one owner.
__device__ __forceinline__ uint32_t seq_bound(const AttnDev &a, uint32_t b) {
    if (b == 0) return 0u;
    const int32_t c = __ldg(a.cu + b);
    return c < 0 ? 0u : min(uint32_t(c), a.n_tokens);
}

// Which block of ROWS rows of which sequence a CTA works on.  Block indices are dealt out by height: a block of height u
// sees u key tiles (or, for a key tile, is seen by u query tiles), and the highest come first, so that the last
// CTAs to start are the short ones.  The job's height and sequence follow from cu_seqlens alone: the
// number of blocks of height >= u is  F(u) = sum_b max(0, blocks_b - u + 1), found by bisection over u by a
// warp whose lanes hold the sequences.  Beyond kRankedSeqs sequences, and where entries are out of order, every sequence gets
// the indices  start/ROWS + b ... instead: at least as many as it has blocks (some stay empty), and one bisection.  Forward and backward
// of 12 heads, ranked against in the pack's order: 16 sequences of about 1000 tokens 645 us against 766, 128 of about
// 150 613 against 651, 256 of about 100 503 against 498, 1024 of 32 1682 against 1092.
// Rows behind the last sequence come last.
constexpr uint32_t kRankedSeqs = 192;
// Whether blocks are dealt out by height (whole warps).
__device__ __forceinline__ bool is_ranked(const AttnDev &a) {
    if (a.n_seqs > kRankedSeqs) return false;
    bool falls = false;
    for (uint32_t i = threadIdx.x & 31; i < a.n_seqs; i += 32) falls |= seq_bound(a, i) > seq_bound(a, i + 1);
    return !__any_sync(0xFFFFFFFFu, falls);
}
// Where the rows behind the last sequence begin.
__device__ __forceinline__ uint32_t tail_start(const AttnDev &a) {
    uint32_t from = 0;
    for (uint32_t lo = 0; lo < a.n_seqs;) {
        lo = (lo + a.n_seqs + 1) / 2;
        from = max(from, seq_bound(a, lo));
    }
    return from;
}
struct Job {
    uint32_t first, len;   // the sequence (or the rows behind the last one)
    uint32_t block;        // which block of it
    bool tail, none;
};
template <int ROWS, bool HIGH_IS_LATE>
__device__ __forceinline__ Job find_job(const AttnDev &a, bool ranked, uint32_t index, uint32_t count) {   // whole warps
    const uint32_t all = 0xFFFFFFFFu, lane = threadIdx.x & 31, n = a.n_seqs;
    Job job;
    job.tail = job.none = false;
    uint32_t b, end;
    if (ranked) {
        auto blocks_of = [&](uint32_t i) {
            if (i >= n) return 0u;
            const uint32_t from = seq_bound(a, i), to = seq_bound(a, i + 1);
            return to > from ? (to - from + ROWS - 1) / ROWS : 0u;
        };
        const uint32_t mine = blocks_of(lane);   // the first 32 sequences stay in registers
        uint32_t most = mine;
        for (uint32_t i = lane + 32; i < n; i += 32) most = max(most, blocks_of(i));
        most = __reduce_max_sync(all, most);
        auto at_least = [&](uint32_t u) {
            uint32_t f = mine >= u ? mine - u + 1 : 0u;
            for (uint32_t i = lane + 32; i < n; i += 32) {
                const uint32_t m = blocks_of(i);
                f += m >= u ? m - u + 1 : 0u;
            }
            return __reduce_add_sync(all, f);
        };
        const uint32_t total = at_least(1);
        if (index >= total) {
            job.tail = true;
            b = n;
            job.block = index - total;
        } else {
            uint32_t lo = 1, hi = most;   // the largest u with F(u) > index
            while (lo < hi) {
                const uint32_t mid = (lo + hi + 1) / 2;
                if (at_least(mid) > index) lo = mid;
                else hi = mid - 1;
            }
            uint32_t k = index - at_least(lo + 1);   // among the sequences of lo blocks or more, the k-th
            b = 0;
            for (uint32_t i0 = 0; i0 < n; i0 += 32) {
                const uint32_t m = i0 == 0 ? mine : blocks_of(i0 + lane);
                const uint32_t here = __ballot_sync(all, m >= lo);
                const uint32_t got = __popc(here);
                if (k < got) {   // the lane with k others before it
                    const bool it = (here >> lane & 1u) && __popc(here & ((1u << lane) - 1u)) == k;
                    b = i0 + __ffs(__ballot_sync(all, it)) - 1;
                    break;
                }
                k -= got;
            }
            job.block = lo - 1;
        }
        job.first = seq_bound(a, b);
        end = job.tail ? a.n_tokens : seq_bound(a, b + 1);
    } else {
        const uint32_t slot = HIGH_IS_LATE ? count - 1 - index : index;
        uint32_t lo = 0, hi = n;   // the last b with start(b)/ROWS + b <= slot
        job.first = 0;
        end = a.n_tokens;
        while (lo < hi) {
            const uint32_t mid = (lo + hi + 1) / 2, cut = min(max(seq_bound(a, mid), job.first), end);   // start(mid)
            if (cut / ROWS + mid <= slot) {
                lo = mid;
                job.first = cut;
            } else {
                hi = mid - 1;
                end = cut;
            }
        }
        b = lo;
        job.tail = b == n;
        job.block = slot - (job.first / ROWS + b);
    }
    job.len = end - job.first;
    const uint32_t blocks = (job.len + ROWS - 1) / ROWS;
    job.none = job.block >= blocks;
    if (!HIGH_IS_LATE && !job.tail && !job.none && ranked) job.block = blocks - 1 - job.block;
    return job;
}
inline uint32_t job_count(uint32_t n_tokens, uint32_t n_seqs, uint32_t rows) { return n_tokens / rows + n_seqs + 1; }

// The grid has one CTA per possible job (highest first, heads fastest), but a CTA that has started takes over jobs whose
// CTA has not (cluster launch control), so that the loads and first products of one job run while the rows of the last
// are written, and no barrier, tensor memory or pipeline is set up twice.  One warp asks for the next job as soon as
// the current one has begun, and tells the others.
enum JobKind : uint32_t { kJobNone = 0, kJobWork = 1, kJobTail = 2, kJobStop = 3 };
struct JobWord {
    uint32_t first, len, block, kind, head;
};
template <int ROWS, bool HIGH_IS_LATE>
__device__ __forceinline__ JobWord job_at(const AttnDev &a, bool ranked, uint32_t index, uint32_t heads) {   // whole warps
    const Job j = find_job<ROWS, HIGH_IS_LATE>(a, ranked, index / heads, gridDim.x / heads);
    JobWord w;
    w.first = j.first;
    w.len = j.len;
    w.block = j.block;
    w.head = index % heads;
    w.kind = j.none ? kJobNone : j.tail ? kJobTail : kJobWork;
    return w;
}
struct Jobs {
    uint32_t word, answer, full, empty, asked;   // shared memory addresses; `readers` warps read every job
    uint32_t limit;
    __device__ __forceinline__ Jobs(uint32_t at, uint32_t wait_limit)
        : word(at), answer(at + 16), full(at + 32), empty(at + 40), asked(at + 48), limit(wait_limit) {}
    static constexpr uint32_t kBytes = 64;
    __device__ __forceinline__ void init(uint32_t readers) const {
        mbar_init(full, 1);
        mbar_init(empty, readers);
        mbar_init(asked, 1);
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(word), "r"(0) : "memory");
    }
    // The warp that hands the jobs out: from this CTA's own index on, until there is none left.  AFTER_PREVIOUS: the readers do
    // not get through their first job before the kernel before this one has ended.
    template <int ROWS, bool HIGH_IS_LATE, bool AFTER_PREVIOUS>
    __device__ __forceinline__ bool run(const AttnDev &a, bool ranked, uint32_t heads) const {
        const uint32_t lane = threadIdx.x & 31;
        int index = int(blockIdx.x);
        uint32_t given = 0, questions = 0;
        while (true) {
            JobWord w;
            w.first = w.len = w.block = w.head = 0;
            w.kind = kJobStop;
            if (index >= 0) w = job_at<ROWS, HIGH_IS_LATE>(a, ranked, uint32_t(index), heads);
            if (w.kind != kJobNone) {
                if (lane == 0) {
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(word), "r"(w.first), "r"(w.len), "r"(w.block), "r"(w.kind | (w.head << 2)) : "memory");
                    mbar_arrive(full);
                }
                if (w.kind == kJobStop) return true;
                if (AFTER_PREVIOUS && given == 0) wait_for_previous();
                if (!warp_wait(empty, given & 1, limit)) return false;   // all have begun it
                ++given;
            }
            if (lane == 0) {
                mbar_expect(asked, 16);
                ask_next_cta(answer, asked);
            }
            if (!warp_wait(asked, questions & 1, limit)) return false;
            ++questions;
            index = next_cta(answer);
            __syncwarp();
            fence_async_shared();   // the answer has been read before the next one overwrites it
        }
    }
    __device__ __forceinline__ bool get_alone(uint32_t k, JobWord *w) const {   // one thread
        if (!mbar_wait(full, k & 1, limit)) return false;
        uint32_t last;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w->first), "=r"(w->len), "=r"(w->block), "=r"(last) : "r"(word) : "memory");
        w->kind = last & 3u;
        w->head = last >> 2;
        mbar_arrive(empty);
        return true;
    }
    __device__ __forceinline__ bool get(uint32_t k, JobWord *w) const {         // whole warp
        if (!warp_wait(full, k & 1, limit)) return false;
        uint32_t last;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w->first), "=r"(w->len), "=r"(w->block), "=r"(last) : "r"(word) : "memory");
        w->kind = last & 3u;
        w->head = last >> 2;
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(empty);
        return true;
    }
};

// A ring of tiles in shared memory, each with a barrier that its copy completes and one that says it may be overwritten.
// One warp fills it; the thread that issues the products empties it.  Both walk it with a Place of their own.
struct Place {
    uint32_t at = 0, phase = 0;   // index and the parity of this round
    template <uint32_t N>
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            phase ^= 1;
        }
    }
};

// Writes zeros over `dim` elements of rows [from, to) of one head, by the first `threads` threads of the CTA: rows that
// belong to no sequence.
__device__ __forceinline__ void fill_rows(const RowsOut &o, uint32_t from, uint32_t to, uint32_t head, uint32_t dim, uint32_t threads) {
    const uint32_t per = dim / 8, n = (to - from) * per;
    for (uint32_t i = threadIdx.x; i < n; i += threads) {
        char *p = o.p + (long long)(from + i / per) * o.token + (long long)head * o.head + (i % per) * 16;
        *reinterpret_cast<uint4 *>(p) = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Writes NaN over the rows, by one warp: what a wait that ran out leaves of a job.
__device__ __forceinline__ void poison_rows(const RowsOut &o, uint32_t from, uint32_t to, uint32_t head, uint32_t dim) {
    const uint32_t per = dim / 8, n = (to - from) * per;
    for (uint32_t i = threadIdx.x & 31; i < n; i += 32) {
        char *p = o.p + (long long)(from + i / per) * o.token + (long long)head * o.head + (i % per) * 16;
        *reinterpret_cast<uint4 *>(p) = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);
    }
}

// Zeroes rows [from, 128) of a tile in shared memory, by the warp that loads it, before the matrix unit is told of it:
// rows behind the sequence belong to others, and their zero weight does not cover a NaN.
template <int SUB>
__device__ __forceinline__ void zero_tile_rows(uint32_t tile, uint32_t from) {
    for (int x = 0; x < SUB; ++x)
        for (uint32_t i = from * 8 + (threadIdx.x & 31); i < kTile * 8; i += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + x * (kTile * 128) + i * 16), "r"(0) : "memory");
    fence_async_shared();
    __syncwarp();
}

// Writes 32 accumulator rows (one per lane) as bfloat16 rows, by one warp: COLS columns at a time go through 64 COLS bytes
// of shared memory, so that COLS/8 lanes write one row's COLS columns together.  Written straight from the lanes, 32
// rows at a time, the same stores take 4800 cycles for a tile of 128 x 128 instead of 900.
template <int DP, int COLS>
__device__ __forceinline__ void store_rows(uint32_t stage, uint32_t tmem, float f, const RowsOut &o, uint32_t token, uint32_t head,
                                           uint32_t rows, uint32_t dim) {
    constexpr uint32_t kPer = COLS / 8, kSpread = 8 / kPer;   // 16-byte pieces of a row; rows that share a bank line
    const uint32_t lane = threadIdx.x & 31;
    char *out = o.p + (long long)token * o.token + (long long)head * o.head;
#pragma unroll 1
    for (uint32_t col = 0; col < DP; col += COLS) {
#pragma unroll
        for (int h = 0; h < COLS / 32; ++h) {
            uint32_t x[32];
            tmem_ld32(x, tmem + col + 32 * h);
            tmem_wait_ld();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *v = reinterpret_cast<const float *>(x + 8 * u);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                             ::"r"(stage + lane * (COLS * 2) + (((4 * h + u) ^ ((lane / kSpread) % kPer)) * 16)), "r"(bf16x2(v[0] * f, v[1] * f)),
                               "r"(bf16x2(v[2] * f, v[3] * f)), "r"(bf16x2(v[4] * f, v[5] * f)), "r"(bf16x2(v[6] * f, v[7] * f)) : "memory");
            }
        }
        __syncwarp();
        const uint32_t c = lane % kPer;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) {
            const uint32_t r = i * (32 / kPer) + lane / kPer;
            uint4 v;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                         : "r"(stage + r * (COLS * 2) + ((c ^ ((r / kSpread) % kPer)) * 16)) : "memory");
            if (r < rows && col + 8 * c < dim) *reinterpret_cast<uint4 *>(out + (long long)r * o.token + (col + 8 * c) * 2) = v;
        }
        __syncwarp();
    }
}
// The same as binary32 rows `pitch` elements apart, 16 columns (2 KB of shared memory) at a time.
template <int DP>
__device__ __forceinline__ void store_rows_f32(uint32_t stage, uint32_t tmem, float f, float *out, size_t pitch, uint32_t rows, uint32_t dim) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll 1
    for (uint32_t col = 0; col < DP; col += 16) {
        uint32_t x[16];
        tmem_ld16(x, tmem + col);
        tmem_wait_ld();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float *v = reinterpret_cast<const float *>(x + 4 * u);
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 64 + ((u ^ ((lane / 2) % 4)) * 16)),
                         "f"(v[0] * f), "f"(v[1] * f), "f"(v[2] * f), "f"(v[3] * f) : "memory");
        }
        __syncwarp();
        const uint32_t c = lane % 4;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t r = i * 8 + lane / 4;
            float4 v;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                         : "r"(stage + r * 64 + ((c ^ ((r / 2) % 4)) * 16)) : "memory");
            if (r < rows && col + 4 * c < dim) *reinterpret_cast<float4 *>(out + r * pitch + col + 4 * c) = v;
        }
        __syncwarp();
    }
}

// d = a b^T over DP columns, both operands in shared memory, rows along the result.
template <int DP>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
    const uint32_t da = smem_desc(a, 0), db = smem_desc(b, 0);
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        const uint32_t off = ((i / 4) * (kTile * 128) + (i % 4) * 32) / 16;
        mma_ss(d, da + off, db + off, idesc, i > 0);
    }
}
// d (+)= a b with a (128 bfloat16 columns) in tensor memory, its second half HALF words behind the first, and b in
// shared memory, rows along the summed dimension.
template <int HALF>
__device__ __forceinline__ void product_cols(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    const uint32_t db = smem_desc(b, kTile * 128);
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) mma_ts(d, a + (i / 4) * HALF + (i % 4) * 8, db + i * (2048 / 16), idesc, add || i > 0);
}

// ------------------------------------------------------------------- forward
//
// One CTA: two query tiles of 128 rows (256 consecutive rows of one sequence and head) against the key and
// value tiles up to the diagonal.  Per key tile and query tile:
//     S = Q K^T   (tcgen05, operands in shared memory, S in tensor memory)
//     P = exp2(c S - c m)   by 128 threads, one row each; P goes back to tensor memory as bfloat16, over S
//     O += P V    (tcgen05, P from tensor memory, V from shared memory, O stays in tensor memory)
// m is the largest score a row had when it was last rescaled: O and the row sum are rescaled only when a score
// exceeds it by more than 2^8 after scaling, so P stays below 256 and the rescaling, which has to wait for the products
// in flight, is rare.  The two tiles alternate: while one tile's products run on the tensor cores the other tile's
// exponentials are taken.
// Warps: 0-3 and 4-7 the rows of the two tiles, 8 issues the products, 9 the TMA loads, 10 finds the jobs; 11 only makes
// the third warpgroup whole, which hands registers over to the first two, so that a row of 128 scores stays in registers.
// (The compiler plans with the 168 of the launch and spills 48 bytes at DP = 64 and 108 at 128 beside it.)
//
// Per key tile and query tile the tensor cores need 1024 cycles, the exponentials as many on the 16-wide special function
// unit, and the way from a finished S to the next (scores out of tensor memory, maximum, exponentials, P back, two
// products, four barriers) takes about 3700; two tiles in turn make that 1850 each.  One query tile of 128 rows per CTA and two
// CTAs per SM would hide it too, but read every key and value tile twice.  Measured in ten calls after a pause and in a
// second of calls on end, which meets the power cap: one sequence of 16384 tokens, 12/2 heads x 128, 636 us = 1.30 PFLOP/s
// (0.77 of cuBLAS's best rate) and 720 us = 1.15 (0.80 of its rate under the cap); 12384 tokens in four sequences, 28/4
// heads, 265 us = 1.12 and 301; 8192 tokens in eight sequences, 12/2 heads, 53 us = 0.66 on end: there a CTA has three
// jobs of 7 key tiles, and each starts with a load, a product and a full softmax that nothing hides.

template <int DP>
struct Fwd {
    static constexpr int kSub = DP / 64;                     // 64-wide blocks of a row
    static constexpr int kBytes = kTile * DP * 2;            // one tile
    static constexpr int kStages = DP == 128 ? 4 : 8;        // key and value tiles in flight
    static constexpr int kStageBytes = 4096;                 // per warp, on the way out
    static constexpr int kThreads = 384;
    static constexpr int kRegs = 168, kRowRegs = 200, kOtherRegs = 104;   // at launch; then two warpgroups, one
    static_assert(2 * kRowRegs + kOtherRegs <= 3 * kRegs, "shares of the launch's registers");
    static constexpr int kSmem = 1024 + (2 + kStages) * kBytes + 8 * kStageBytes + 512;
};

template <int DP>
__global__ void __launch_bounds__(Fwd<DP>::kThreads, 1)
attn_forward_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, const __grid_constant__ AttnDev a) {
    using C = Fwd<DP>;
    extern __shared__ char smem_raw[];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = a.q_heads / a.kv_heads;
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t sq = base, sring = base + 2 * C::kBytes;
    const uint32_t stage = sring + C::kStages * C::kBytes, bars = stage + 8 * C::kStageBytes;
    const Jobs jobs(bars, a.wait_limit);
    const uint32_t q_full = bars + Jobs::kBytes, q_empty = q_full + 8, s_full = q_full + 16, p_full = q_full + 32, o_full = q_full + 48,
                   raw = q_full + 64, full = q_full + 72, empty = full + 8 * C::kStages,
                   tmem_slot = empty + 8 * C::kStages;

    if (warp == 8) tmem_alloc(tmem_slot, 512);
    if (threadIdx.x == 0) {
        jobs.init(10);
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        mbar_init(raw, 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(s_full + 8 * t, 1);
            mbar_init(p_full + 8 * t, 4);
            mbar_init(o_full + 8 * t, 1);
        }
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        fence_barrier_init();
    }
    const bool ranked = warp == 10 && is_ranked(a);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    bool ok = true;
    JobWord w;
    w.kind = kJobNone;

    if (warp >= 8) {
        registers_down<C::kOtherRegs>();
        if (warp == 9) {   // -------------------------------------------- loads
            uint32_t tiles = 0, fixed = 0, n = 0;   // jobs, tiles with rows of others, ring items so far
            Place at;
            for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
                if (w.kind != kJobWork) continue;
                const uint32_t row0 = w.block * 2 * kTile, kv_head = w.head / group;
                const bool two = row0 + kTile < w.len;
                const uint32_t items = 2 * (w.block * 2 + 1 + (two ? 1 : 0));
                if (tiles > 0 && !(ok = warp_wait(q_empty, (tiles - 1) & 1, a.wait_limit))) break;
                ++tiles;
                if (lane == 0) {
                    mbar_expect(q_full, (two ? 2 : 1) * C::kBytes);
                    for (int t = 0; t < (two ? 2 : 1); ++t)
                        for (int x = 0; x < C::kSub; ++x)
                            tma_load(sq + t * C::kBytes + x * (kTile * 128), &mq, q_full, x * 64, int(w.head) * a.q_mul,
                                     int(w.first + row0 + t * kTile));
                }
                for (uint32_t i = 0; i < items; ++i, ++n, at.template next<C::kStages>()) {   // K, V, K, V, ...
                    if (n >= C::kStages && !(ok = warp_wait(empty + 8 * at.at, at.phase ^ 1, a.wait_limit))) break;
                    const bool is_k = (i & 1) == 0, ragged = !is_k && w.len < (i / 2 + 1) * kTile;
                    const uint32_t tile = sring + at.at * C::kBytes, bar = ragged ? raw : full + 8 * at.at;
                    if (lane == 0) {
                        mbar_expect(bar, C::kBytes);
                        for (int x = 0; x < C::kSub; ++x)
                            tma_load(tile + x * (kTile * 128), is_k ? &mk : &mv, bar, x * 64, int(kv_head) * (is_k ? a.k_mul : a.v_mul),
                                     int(w.first + (i / 2) * kTile));
                    }
                    if (ragged) {
                        if (!(ok = warp_wait(raw, fixed & 1, a.wait_limit))) break;
                        ++fixed;
                        zero_tile_rows<C::kSub>(tile, w.len - (i / 2) * kTile);
                        if (lane == 0) mbar_arrive(full + 8 * at.at);
                    }
                }
                if (!ok) break;
            }
            // the CTA must not end, nor its memory be given back, before the last loads and releases have arrived
            if (tiles > 0) {
                mbar_wait(q_full, (tiles - 1) & 1, a.wait_limit);
                if (ok) ok = warp_wait(q_empty, (tiles - 1) & 1, a.wait_limit);
            }
            for (uint32_t i = n > C::kStages ? n - C::kStages : 0; i < n; ++i) {
                mbar_wait(full + 8 * (i % C::kStages), (i / C::kStages) & 1, a.wait_limit);
                if (ok) ok = warp_wait(empty + 8 * (i % C::kStages), (i / C::kStages) & 1, a.wait_limit);
            }
        } else if (warp == 8) {   // --------------------------------- products
            // One thread: between two batches of products the tensor cores hold about one product's work, so every
            // cycle spent here in between is one that they may lose.  Spinning for P instead of sleeping gains 3 %
            // here, and costs the backward kernels 3 %, whose row warps are the busier ones.
            if (lane == 0) {
                const uint32_t id_s = mma_desc(kTile, false) | a.negate, id_o = mma_desc(DP, true);
                uint32_t tiles = 0, done0 = 0, done1 = 0;   // jobs, blocks of the first and second tile so far
                Place at;   // of the oldest ring item not yet released
                auto tile_of = [&](const Place &p) { return sring + p.at * C::kBytes; };
                auto wait_tile = [&](const Place &p) { return mbar_wait(full + 8 * p.at, p.phase, a.wait_limit); };
                auto release = [&]() {
                    mma_commit(empty + 8 * at.at);
                    at.template next<C::kStages>();
                };
                for (uint32_t k = 0; (ok = jobs.get_alone(k, &w)) && w.kind != kJobStop; ++k) {
                    if (w.kind != kJobWork) continue;
                    const bool two = w.block * 2 * kTile + kTile < w.len;
                    const uint32_t nb0 = w.block * 2 + 1, nb = nb0 + (two ? 1 : 0);   // key tiles of the first tile; of both
                    if (!(ok = mbar_wait(q_full, tiles & 1, a.wait_limit) && wait_tile(at))) break;
                    ++tiles;
                    tc_fence_after();
                    product_rows<DP>(tmem, sq, tile_of(at), id_s);   // S_0 = Q_0 K^T
                    mma_commit(s_full);
                    if (two) {
                        product_rows<DP>(tmem + 128, sq + C::kBytes, tile_of(at), id_s);
                        mma_commit(s_full + 8);
                    }
                    release();
                    if (nb == 1) mma_commit(q_empty);
                    for (uint32_t j = 0; j < nb; ++j) {
                        const Place v = at;
                        Place key = at;
                        key.template next<C::kStages>();
                        if (!(ok = wait_tile(v) && (j + 1 == nb || wait_tile(key)))) break;
                        if (j < nb0) {
                            if (!(ok = mbar_spin(p_full, done0 & 1, a.wait_limit))) break;
                            ++done0;
                            tc_fence_after();
                            product_cols<32>(tmem + 256, tmem, tile_of(v), id_o, j > 0);   // O_0 += P_0 V
                            mma_commit(o_full);
                            if (j + 1 < nb0) {
                                product_rows<DP>(tmem, sq, tile_of(key), id_s);
                                mma_commit(s_full);
                            }
                        }
                        if (two) {
                            if (!(ok = mbar_spin(p_full + 8, done1 & 1, a.wait_limit))) break;
                            ++done1;
                            tc_fence_after();
                            product_cols<32>(tmem + 384, tmem + 128, tile_of(v), id_o, j > 0);
                            mma_commit(o_full + 8);
                            if (j + 1 < nb) {
                                product_rows<DP>(tmem + 128, sq + C::kBytes, tile_of(key), id_s);
                                mma_commit(s_full + 8);
                            }
                        }
                        release();
                        if (j + 1 < nb) {
                            release();
                            if (j + 2 == nb) mma_commit(q_empty);   // the last use of Q
                        }
                    }
                    if (!ok) break;
                }
            }
        } else if (warp == 10) {   // ------------------------------------ jobs
            ok = jobs.template run<2 * kTile, true, false>(a, ranked, a.q_heads);
        }
    } else {   // ------------------------------------------- a row of a tile
        registers_up<C::kRowRegs>();
        const int t = warp >> 2;
        const uint32_t lanes = (warp & 3) << 21;   // tensor memory lane 32 (warp & 3)
        const uint32_t ts = tmem + t * 128 + lanes, to = tmem + 256 + t * 128 + lanes;
        const uint32_t local = (warp & 3) * 32 + lane;
        const float c = a.exp2_scale;
        uint32_t it = 0;   // row blocks of this tile so far
        for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
            const uint32_t row0 = w.block * 2 * kTile;
            if (w.kind == kJobTail) {
                const uint32_t from = w.first + row0, end = min(w.first + w.len, from + 2 * kTile);
                fill_rows(a.o, from, end, w.head, a.head_dim, 256);
                for (uint32_t i = from + threadIdx.x; i < end; i += 256) a.lse[size_t(w.head) * a.n_tokens + i] = -INFINITY;
            }
            if (w.kind != kJobWork || row0 + t * kTile >= w.len) continue;
            const uint32_t my_blocks = w.block * 2 + 1 + t;
            float m = -INFINITY;
            float2 sum = make_float2(0.f, 0.f);
            for (uint32_t j = 0; j < my_blocks; ++j, ++it) {
                if (!(ok = warp_wait(s_full + 8 * t, it & 1, a.wait_limit))) break;
                tc_fence_after();
                uint32_t r[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_ld32(r[i], ts + 32 * i);
                tmem_wait_ld();
                if (j == my_blocks - 1) {   // the diagonal tile
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (uint32_t(i) > local) r[i / 32][i % 32] = __float_as_uint(-INFINITY);
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 128; i += 2)
                    mx[(i / 2) % 4] = max3_nan(mx[(i / 2) % 4], __uint_as_float(r[i / 32][i % 32]), __uint_as_float(r[i / 32][i % 32 + 1]));
                float top = max3_nan(max3_nan(mx[0], mx[1], mx[1]), mx[2], mx[3]);
                top += top - top;   // an infinite score, like a NaN, makes its whole row NaN
                if (j == 0) m = top;
                else if (__any_sync(0xFFFFFFFFu, !((top - m) * c <= 8.0f))) {
                    if (!(ok = warp_wait(o_full + 8 * t, (it - 1) & 1, a.wait_limit))) break;
                    tc_fence_after();
                    const float next = max3_nan(m, top, top), f = exp2_approx((m - next) * c);
                    sum = mul2(sum, make_float2(f, f));
                    m = next;
#pragma unroll 1
                    for (int i = 0; i < DP / 16; ++i) {   // rare: few registers matter more than speed
                        uint32_t x[16];
                        tmem_ld16(x, to + 16 * i);
                        tmem_wait_ld();
#pragma unroll
                        for (int u = 0; u < 16; ++u) x[u] = __float_as_uint(__uint_as_float(x[u]) * f);
                        tmem_st16(to + 16 * i, x);
                    }
                }
                const float2 c2 = make_float2(c, c), mc = make_float2(-m * c, -m * c);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = fma2(make_float2(__uint_as_float(r[h][2 * i]), __uint_as_float(r[h][2 * i + 1])), c2, mc);
                        const float2 e = make_float2(exp2_approx(x.x), exp2_approx(x.y));
                        sum = add2(sum, e);
                        p[i] = bf16x2(e.x, e.y);
                    }
                    tmem_st16(ts + 16 * h, p);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * t);
            }
            if (!ok || !(ok = warp_wait(o_full + 8 * t, (it - 1) & 1, a.wait_limit))) break;
            tc_fence_after();
            const float total = sum.x + sum.y, inv = 1.0f / total;
            const uint32_t row = row0 + t * kTile + local;
            if (row < w.len) a.lse[size_t(w.head) * a.n_tokens + w.first + row] = m * fabsf(a.scale) + logf(total);
            const uint32_t row_w = row - lane;   // the warp's first row
            store_rows<DP, 64>(stage + warp * C::kStageBytes, to, inv, a.o, w.first + row_w, w.head, w.len > row_w ? w.len - row_w : 0u, a.head_dim);
            tc_fence_before();   // O has been read: the next job's first product, after this warp's next arrival, may overwrite it
        }
    }
    tc_fence_before();
    const bool bad = __syncthreads_or(!ok);
    tc_fence_after();
    if (warp == 8) tmem_free(tmem, 512);
    if (bad) {
        if (w.kind == kJobWork) {   // each warp's own last job
            const uint32_t from = w.first + w.block * 2 * kTile, end = min(w.first + w.len, from + 2 * kTile);
            poison_rows(a.o, from, end, w.head, a.head_dim);
            for (uint32_t i = from + lane; i < end; i += 32) a.lse[size_t(w.head) * a.n_tokens + i] = __int_as_float(0x7FFFFFFF);
        }
        if (threadIdx.x == 0) atomicAdd(&g_attn_faults, 1u);
    }
}

// ------------------------------------------------------------------- backward
//
// With P = exp2(c S - log2(e) lse) and the row term D_i = sum_d dO_id O_id = sum_j P_ij dP_ij:
//     dV = P^T dO,   dP = dO V^T,   dS = P (dP - D),   dQ = scale dS K,   dK = scale dS^T Q
// The row term comes from the rounded O first.  A row of dS adds up to what that was off by, so the kernel for dQ, which
// has the whole row, leaves a better one for the other; and rows that see one key tile alone, where O is largest and
// its rounding tells most, take the second form from the start.
// One kernel sums over the query tiles for a key tile (dK, dV), the other over the key tiles for a query tile
// (dQ).  Both make S and dP again, seven products in all where five would do with dQ added up in memory by
// atomics; in return every sum has one owner and one order, and two calls give the same bits.

// The row terms: a half warp per row and head, four of them in flight.
constexpr int kRowThreads = 256, kRowsInFlight = 4;
static __global__ void __launch_bounds__(kRowThreads) attn_rows_kernel(const __grid_constant__ AttnDev a) {
    let_next_start();
    const uint32_t first = blockIdx.x * (kRowThreads / 16 * kRowsInFlight) + threadIdx.x / 16, l = threadIdx.x & 15;
    uint4 x[kRowsInFlight], y[kRowsInFlight];
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
        const uint32_t unit = first + i * (kRowThreads / 16), head = unit % a.q_heads, t = unit / a.q_heads;
        x[i] = y[i] = make_uint4(0u, 0u, 0u, 0u);
        if (t < a.n_tokens && l * 8 < a.head_dim) {
            x[i] = *reinterpret_cast<const uint4 *>(a.o.p + (long long)t * a.o.token + (long long)head * a.o.head + l * 16);
            y[i] = *reinterpret_cast<const uint4 *>(a.do_in + (long long)t * a.do_token + (long long)head * a.do_head + l * 16);
        }
    }
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
        const uint32_t unit = first + i * (kRowThreads / 16), head = unit % a.q_heads, t = unit / a.q_heads;
        const uint32_t xs[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, ys[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            s = fmaf(__uint_as_float(xs[u] << 16), __uint_as_float(ys[u] << 16), s);
            s = fmaf(__uint_as_float(xs[u] & 0xFFFF0000u), __uint_as_float(ys[u] & 0xFFFF0000u), s);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (t < a.n_tokens && l == 0) {
            const size_t at = size_t(head) * a.n_tokens + t;
            a.rows[at] = make_float2(-kLog2e * a.lse[at], s);
        }
    }
}

// One CTA: one key tile of a key head, over the query tiles from the diagonal to the end of the sequence, for the query
// heads of the group (or of one part of it).  Rows of the accumulators are keys, so P^T and dS^T come out of
// the products as they have to go into the next ones, from tensor memory; nothing is transposed.
// Warps: 0-3 and 4-7 take the two halves of the query columns, 8 issues the products, 9 the TMA loads, 10 fetches the
// row terms, 11 finds the jobs.  While the threads make dS of one query tile the tensor cores run dV and the next S;
// while they take the next exponentials, dK and the next dP.
//
// Four products of 512 cycles per query tile; a turn takes about 3400, the way from S through P, dV and the next S:
// tensor memory (512 columns: S, dP, dV, dK) has no room for a second S at head sizes above 64 (up to 64, dV and dK take 64
// columns each and it would fit; the same code serves both), and the two loads of 32 KB per turn take about 2200 cycles
// each with shared memory for two turns.  Measured: 12384 tokens, 28/4 heads x 128, 584 us (1.02 PFLOP/s of the four
// products done).
template <int DP>
struct BwdKv {
    static constexpr int kSub = DP / 64;
    static constexpr int kBytes = kTile * DP * 2;
    static constexpr int kStages = DP == 128 ? 4 : 8, kPairs = kStages / 2;
    static constexpr int kRowSlots = 4;
    static constexpr int kStageBytes = 2048;   // per warp, on the way out
    static constexpr int kThreads = 384;
    static constexpr int kRegs = 168, kRowRegs = 192, kOtherRegs = 120;   // at launch; then two warpgroups, one
    static_assert(2 * kRowRegs + kOtherRegs <= 3 * kRegs, "shares of the launch's registers");
    static constexpr int kSmem = 1024 + (2 + kStages) * kBytes + kRowSlots * 1024 + 8 * kStageBytes + 512;
};

template <int DP>
__global__ void __launch_bounds__(BwdKv<DP>::kThreads, 1)
attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ AttnDev a) {
    using C = BwdKv<DP>;
    extern __shared__ char smem_raw[];
    const uint32_t lots = a.kv_heads * a.parts;   // a job's head names the key head and the part of its group
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t heads = a.q_heads / a.kv_heads / a.parts;
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t sk = base, sv = base + C::kBytes, sring = base + 2 * C::kBytes;
    const uint32_t srows = sring + C::kStages * C::kBytes;   // per slot: 128 x -log2(e) lse, 128 x D
    const uint32_t stage = srows + C::kRowSlots * 1024, bars = stage + 8 * C::kStageBytes;
    const Jobs jobs(bars, a.wait_limit);
    const uint32_t kv_full = bars + Jobs::kBytes, kv_empty = kv_full + 8, s_full = kv_full + 16, dp_full = kv_full + 24, p_full = kv_full + 32,
                   ds_full = kv_full + 40, done = kv_full + 48, raw = kv_full + 56, rows_full = kv_full + 64, rows_empty = rows_full + 8 * C::kRowSlots,
                   full = rows_empty + 8 * C::kRowSlots, empty = full + 8 * C::kStages, tmem_slot = empty + 8 * C::kStages;

    let_next_start();
    if (warp == 8) tmem_alloc(tmem_slot, 512);
    if (threadIdx.x == 0) {
        jobs.init(11);
        mbar_init(kv_full, 1);
        mbar_init(kv_empty, 1);
        mbar_init(raw, 1);
        mbar_init(s_full, 1);
        mbar_init(dp_full, 1);
        mbar_init(p_full, 8);
        mbar_init(ds_full, 8);
        mbar_init(done, 1);
        for (int i = 0; i < C::kRowSlots; ++i) {
            mbar_init(rows_full + 8 * i, 1);
            mbar_init(rows_empty + 8 * i, 8);
        }
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        fence_barrier_init();
    }
    const bool ranked = warp == 11 && is_ranked(a);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    const uint32_t t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 384;
    bool ok = true;
    JobWord w;
    w.kind = kJobNone;
    // A pair of places takes Q and dO of a query tile, by turns the one way and the other: dO is done with first, and the
    // tile that is wanted first two tiles later, a Q, goes where it was.
    auto q_slot = [](const Place &p) { return 2 * p.at + p.phase; };
    auto g_slot = [](const Place &p) { return 2 * p.at + (p.phase ^ 1); };
    auto q_tiles_of = [](const JobWord &j) { return (j.len + kTile - 1) / kTile - j.block; };   // from the diagonal on
    // Row terms come from the kernel before: whoever depends on them, through others' work too, waits for its end first, so
    // that a limited wait is only ever for this CTA.
    auto get_job = [&](uint32_t k) {
        if (k == 1) wait_for_previous();
        return jobs.get(k, &w);
    };
    auto kv_head_of = [&](const JobWord &j) { return j.head % a.kv_heads; };
    auto head0_of = [&](const JobWord &j) { return kv_head_of(j) * (a.q_heads / a.kv_heads) + (j.head / a.kv_heads) * heads; };

    if (warp >= 8) {
        registers_down<C::kOtherRegs>();
        if (warp == 9) {   // -------------------------------------------- loads
            uint32_t tiles = 0, fixed = 0, n = 0;   // jobs, tiles with rows of others, query tiles so far
            Place at;
            for (uint32_t k = 0; (ok = get_job(k)) && w.kind != kJobStop; ++k) {
                if (w.kind != kJobWork) continue;
                if (tiles > 0 && !(ok = warp_wait(kv_empty, (tiles - 1) & 1, a.wait_limit))) break;
                ++tiles;
                const uint32_t q_tiles = q_tiles_of(w), kv_head = kv_head_of(w);
                if (lane == 0) {
                    mbar_expect(kv_full, 2 * C::kBytes);
                    for (int x = 0; x < C::kSub; ++x) {
                        tma_load(sk + x * (kTile * 128), &mk, kv_full, x * 64, int(kv_head) * a.k_mul, int(w.first + w.block * kTile));
                        tma_load(sv + x * (kTile * 128), &mv, kv_full, x * 64, int(kv_head) * a.v_mul, int(w.first + w.block * kTile));
                    }
                }
                uint32_t h = head0_of(w), i = w.block;
                for (uint32_t u = 0; ok && u < heads * q_tiles; ++u, ++n, at.template next<C::kPairs>()) {
                    const bool ragged = w.len < (i + 1) * kTile;
                    if (n == C::kPairs) wait_for_previous();
                    for (uint32_t which = 0; which < 2; ++which) {   // Q, dO
                        const bool is_q = which == 0;
                        const uint32_t slot = is_q ? q_slot(at) : g_slot(at), tile = sring + slot * C::kBytes;
                        const uint32_t bar = ragged ? raw : full + 8 * slot;
                        if (n >= C::kPairs && !(ok = warp_wait(empty + 8 * slot, at.phase ^ 1, a.wait_limit))) break;
                        if (lane == 0) {
                            mbar_expect(bar, C::kBytes);
                            for (int x = 0; x < C::kSub; ++x)
                                tma_load(tile + x * (kTile * 128), is_q ? &mq : &mdo, bar, x * 64, int(h) * (is_q ? a.q_mul : a.do_mul),
                                         int(w.first + i * kTile));
                        }
                        if (ragged) {
                            if (!(ok = warp_wait(raw, fixed & 1, a.wait_limit))) break;
                            ++fixed;
                            zero_tile_rows<C::kSub>(tile, w.len - i * kTile);
                            if (lane == 0) mbar_arrive(full + 8 * slot);
                        }
                    }
                    if (++i == w.block + q_tiles) {
                        i = w.block;
                        ++h;
                    }
                }
                if (!ok) break;
            }
            // the CTA must not end, nor its memory be given back, before the last loads and releases have arrived
            if (tiles > 0) {
                mbar_wait(kv_full, (tiles - 1) & 1, a.wait_limit);
                if (ok) ok = warp_wait(kv_empty, (tiles - 1) & 1, a.wait_limit);
            }
            for (uint32_t i = n > C::kPairs ? n - C::kPairs : 0; i < n; ++i)
                for (uint32_t slot = 2 * (i % C::kPairs); slot < 2 * (i % C::kPairs) + 2; ++slot) {
                    mbar_wait(full + 8 * slot, (i / C::kPairs) & 1, a.wait_limit);
                    if (ok) ok = warp_wait(empty + 8 * slot, (i / C::kPairs) & 1, a.wait_limit);
                }
        } else if (warp == 10) {   // -------------------------------- row terms
            wait_for_previous();
            uint32_t n = 0;
            for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
                if (w.kind != kJobWork) continue;
                const uint32_t q_tiles = q_tiles_of(w);
                uint32_t h = head0_of(w), i = w.block;
                for (uint32_t u = 0; u < heads * q_tiles; ++u, ++n) {
                    const uint32_t slot = n % C::kRowSlots, use = n / C::kRowSlots;
                    const float2 *src = a.rows + size_t(h) * a.n_tokens + w.first + i * kTile;
                    float2 v[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        v[x] = i * kTile + lane + 32 * x < w.len ? __ldcg(src + lane + 32 * x) : make_float2(0.f, 0.f);
                    if (use > 0 && !(ok = warp_wait(rows_empty + 8 * slot, (use - 1) & 1, a.wait_limit))) break;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint32_t at = srows + slot * 1024 + (lane + 32 * x) * 4;
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v[x].x) : "memory");
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 512), "f"(v[x].y) : "memory");
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(rows_full + 8 * slot);
                    if (++i == w.block + q_tiles) {
                        i = w.block;
                        ++h;
                    }
                }
                if (!ok) break;
            }
        } else if (warp == 8) {   // --------------------------------- products
            if (lane == 0) {   // one thread, as in the forward kernel
                const uint32_t id_s = mma_desc(kTile, false), id_o = mma_desc(DP, true);
                uint32_t tiles = 0, it = 0;   // jobs, query tiles so far
                Place at;                     // of the query tile at hand
                auto tile_of = [&](uint32_t slot) { return sring + slot * C::kBytes; };
                auto wait_tile = [&](uint32_t slot, const Place &p) { return mbar_wait(full + 8 * slot, p.phase, a.wait_limit); };
                for (uint32_t k = 0; (ok = jobs.get_alone(k, &w)) && w.kind != kJobStop; ++k) {
                    if (k == 0 && w.kind != kJobWork) wait_for_previous();
                    if (w.kind != kJobWork) continue;
                    const uint32_t total = q_tiles_of(w) * heads;
                    if (!(ok = mbar_wait(kv_full, tiles & 1, a.wait_limit) && wait_tile(q_slot(at), at))) break;
                    ++tiles;
                    tc_fence_after();
                    product_rows<DP>(t_s, sk, tile_of(q_slot(at)), id_s | a.negate);   // S^T = K Q^T
                    mma_commit(s_full);
                    if (!(ok = wait_tile(g_slot(at), at))) break;
                    product_rows<DP>(t_dp, sv, tile_of(g_slot(at)), id_s);             // dP^T = V dO^T
                    mma_commit(dp_full);
                    if (total == 1) mma_commit(kv_empty);
                    if (k == 0) wait_for_previous();
                    for (uint32_t u = 0; u < total; ++u, ++it) {
                        const bool more = u + 1 < total;
                        const uint32_t q = q_slot(at), g = g_slot(at);
                        at.template next<C::kPairs>();
                        const uint32_t q_next = q_slot(at), g_next = g_slot(at);
                        if (more && !(ok = wait_tile(q_next, at))) break;
                        if (!(ok = mbar_wait(p_full, it & 1, a.wait_limit))) break;
                        tc_fence_after();
                        product_cols<64>(t_dv, t_s, tile_of(g), id_o, u > 0);     // dV += P^T dO
                        mma_commit(empty + 8 * g);
                        if (more) {
                            product_rows<DP>(t_s, sk, tile_of(q_next), id_s | a.negate);
                            mma_commit(s_full);
                            if (!(ok = wait_tile(g_next, at))) break;
                        }
                        if (!(ok = mbar_wait(ds_full, it & 1, a.wait_limit))) break;
                        tc_fence_after();
                        product_cols<64>(t_dk, t_dp, tile_of(q), id_o, u > 0);    // dK += dS^T Q
                        mma_commit(empty + 8 * q);
                        if (more) {
                            product_rows<DP>(t_dp, sv, tile_of(g_next), id_s);
                            mma_commit(dp_full);
                            if (u + 2 == total) mma_commit(kv_empty);   // the last use of K and V
                        } else {
                            mma_commit(done);
                        }
                    }
                    if (!ok) break;
                }
            }
        } else {   // ------------------------------------------------ jobs
            ok = jobs.template run<kTile, false, true>(a, ranked, lots);
        }
    } else {   // ---------------------- a key row, half of the query columns
        registers_up<C::kRowRegs>();
        wait_for_previous();
        const uint32_t half = warp >> 2, lanes = (warp & 3) << 21, col0 = half * 64;
        const uint32_t local = (warp & 3) * 32 + lane;
        const float2 c2 = make_float2(a.exp2_scale, a.exp2_scale);
        uint32_t it = 0, tiles = 0;
        for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
            const uint32_t kv_head = kv_head_of(w), part = w.head / a.kv_heads;
            if (w.kind == kJobTail && part == 0) {
                const uint32_t from = w.first + w.block * kTile, to = min(w.first + w.len, from + kTile);
                fill_rows(a.d_k, from, to, kv_head, a.head_dim, 256);
                fill_rows(a.d_v, from, to, kv_head, a.head_dim, 256);
            }
            if (w.kind != kJobWork) continue;
            const uint32_t q_tiles = q_tiles_of(w), total = q_tiles * heads, last = (w.len % kTile) ? w.len % kTile : kTile;
            uint32_t tile = 0;   // query tiles behind the diagonal one, of the current head
            for (uint32_t u = 0; u < total; ++u, ++it) {
                const uint32_t slot = it % C::kRowSlots;
                const uint32_t lo = tile == 0 ? local : 0u, hi = tile + 1 == q_tiles ? last : uint32_t(kTile);
                const bool whole = tile != 0 && hi == kTile;   // every query of the tile sees every key of this one
                if (++tile == q_tiles) tile = 0;
                const uint32_t terms = srows + slot * 1024 + col0 * 4;
                if (!(ok = warp_wait(rows_full + 8 * slot, (it / C::kRowSlots) & 1, a.wait_limit))) break;
                if (!(ok = warp_wait(s_full, it & 1, a.wait_limit))) break;
                tc_fence_after();
                float p[64];
                {
                    uint32_t r[2][32];
                    tmem_ld32(r[0], t_s + lanes + col0);
                    tmem_ld32(r[1], t_s + lanes + col0 + 32);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 64; x += 4) {
                        float4 l;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l.x), "=f"(l.y), "=f"(l.z), "=f"(l.w) : "r"(terms + x * 4));
                        const uint32_t *v = &r[x / 32][x % 32];
                        const float2 y = fma2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), c2, make_float2(l.x, l.y));
                        const float2 z = fma2(make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])), c2, make_float2(l.z, l.w));
                        p[x] = exp2_approx(y.x);
                        p[x + 1] = exp2_approx(y.y);
                        p[x + 2] = exp2_approx(z.x);
                        p[x + 3] = exp2_approx(z.y);
                    }
                    if (!whole) {
#pragma unroll
                        for (int x = 0; x < 64; ++x)
                            if (col0 + x < lo || col0 + x >= hi) p[x] = 0.f;
                    }
#pragma unroll
                    for (int x = 0; x < 32; ++x) r[0][x] = bf16x2(p[2 * x], p[2 * x + 1]);
                    tmem_st32(t_s + lanes + col0, r[0]);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
                if (!(ok = warp_wait(dp_full, it & 1, a.wait_limit))) break;
                tc_fence_after();
                {
                    uint32_t r[2][32];
                    tmem_ld32(r[0], t_dp + lanes + col0);
                    tmem_ld32(r[1], t_dp + lanes + col0 + 32);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 64; x += 4) {
                        float4 d;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(d.x), "=f"(d.y), "=f"(d.z), "=f"(d.w) : "r"(terms + 512 + x * 4));
                        const uint32_t *v = &r[x / 32][x % 32];
                        p[x] *= __uint_as_float(v[0]) - d.x;
                        p[x + 1] *= __uint_as_float(v[1]) - d.y;
                        p[x + 2] *= __uint_as_float(v[2]) - d.z;
                        p[x + 3] *= __uint_as_float(v[3]) - d.w;
                    }
                    if (!whole) {
#pragma unroll
                        for (int x = 0; x < 64; ++x)
                            if (col0 + x < lo || col0 + x >= hi) p[x] = 0.f;
                    }
#pragma unroll
                    for (int x = 0; x < 32; ++x) r[0][x] = bf16x2(p[2 * x], p[2 * x + 1]);
                    tmem_st32(t_dp + lanes + col0, r[0]);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(ds_full);
                    mbar_arrive(rows_empty + 8 * slot);
                }
            }
            if (!ok || !(ok = warp_wait(done, tiles & 1, a.wait_limit))) break;
            ++tiles;
            tc_fence_after();
            // the first half of the threads writes dV, the second dK
            const uint32_t row_w = w.block * kTile + local - lane, rows = w.len > row_w ? w.len - row_w : 0u;
            const float f = half ? a.scale : 1.0f;
            const uint32_t acc = (half ? t_dk : t_dv) + lanes;
            if (a.parts > 1)
                store_rows_f32<DP>(stage + warp * C::kStageBytes, acc, f,
                                   a.part_sums + (((size_t(part) * 2 + (1 - half)) * a.n_tokens + w.first + row_w) * a.kv_heads + kv_head) * a.head_dim,
                                   size_t(a.kv_heads) * a.head_dim, rows, a.head_dim);
            else
                store_rows<DP, 32>(stage + warp * C::kStageBytes, acc, f, half ? a.d_k : a.d_v, w.first + row_w, kv_head, rows, a.head_dim);
            tc_fence_before();
        }
    }
    tc_fence_before();
    const bool bad = __syncthreads_or(!ok);
    tc_fence_after();
    if (warp == 8) tmem_free(tmem, 512);
    if (bad) {
        if (w.kind == kJobWork) {   // each warp's own last job
            const uint32_t from = w.first + w.block * kTile, to = min(w.first + w.len, from + kTile);
            const uint32_t kv_head = kv_head_of(w), part = w.head / a.kv_heads;
            if (a.parts > 1)
                for (uint32_t which = 0; which < 2; ++which)
                    for (uint32_t i = lane; i < (to - from) * a.head_dim; i += 32)
                        a.part_sums[(((size_t(part) * 2 + which) * a.n_tokens + from + i / a.head_dim) * a.kv_heads + kv_head) * a.head_dim +
                                    i % a.head_dim] = __int_as_float(0x7FFFFFFF);
            else {
                poison_rows(a.d_k, from, to, kv_head, a.head_dim);
                poison_rows(a.d_v, from, to, kv_head, a.head_dim);
            }
        }
        if (threadIdx.x == 0) atomicAdd(&g_attn_faults, 1u);
    }
}

// Adds the parts of dK and dV in order and rounds them once.
static __global__ void __launch_bounds__(256) attn_sum_parts_kernel(const __grid_constant__ AttnDev a) {
    wait_for_previous();
    const uint32_t per = a.head_dim / 8;
    const size_t rows = size_t(a.n_tokens) * a.kv_heads, n = 2 * rows * per;
    const size_t i = size_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= n) return;
    const uint32_t which = i >= rows * per;   // 0: dK, 1: dV
    const size_t j = i - which * rows * per, row = j / per;
    const uint32_t t = uint32_t(row / a.kv_heads), h = uint32_t(row % a.kv_heads), x = uint32_t(j % per) * 8;
    if (t >= tail_start(a)) return;   // rows of no sequence were written as zero
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (uint32_t part0 = 0; part0 < a.parts; part0 += 4) {
        float4 u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 *src = reinterpret_cast<const float4 *>(a.part_sums + ((size_t(part0 + i) * 2 + which) * rows + row) * a.head_dim + x);
            const bool there = part0 + i < a.parts;
            u[i] = there ? __ldcs(src) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[i] = there ? __ldcs(src + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[0] += u[i].x; s[1] += u[i].y; s[2] += u[i].z; s[3] += u[i].w;
            s[4] += v[i].x; s[5] += v[i].y; s[6] += v[i].z; s[7] += v[i].w;
        }
    }
    const RowsOut &o = which ? a.d_v : a.d_k;
    *reinterpret_cast<uint4 *>(o.p + (long long)t * o.token + (long long)h * o.head + x * 2) =
        make_uint4(bf16x2(s[0], s[1]), bf16x2(s[2], s[3]), bf16x2(s[4], s[5]), bf16x2(s[6], s[7]));
}

// One CTA: two query tiles of 128 rows (256 consecutive rows of one sequence and head) over the key tiles up to the
// diagonal, as in the forward kernel: each key and value tile is loaded once for both.  Tensor memory holds dQ and one
// working place per tile, which takes S, then dP as soon as S has been read, then dS as bfloat16.  The two tiles alternate:
// a tile's threads take its exponentials and make its dS while the tensor cores work for the other.
// Warps: 0-3 and 4-7 the rows of the two tiles, 8 issues the products, 9 the TMA loads, 10 finds the jobs.
//
// Six products of 512 cycles per key tile and pair of query tiles; a turn takes about 4300, of which the issuing thread
// loses some 150 at each of its four waits.  One query tile per CTA with S double-buffered loads twice as much, has room
// for one value tile, and waits for it: 447 us where this took 385 (12384 tokens, 28/4 heads x 128; 358 on a cool card).
template <int DP>
struct BwdQ {
    static constexpr int kSub = DP / 64;
    static constexpr int kBytes = kTile * DP * 2;
    static constexpr int kKeys = DP == 128 ? 2 : 4, kValues = DP == 128 ? 1 : 3, kStages = kKeys + kValues;   // tiles in flight
    static constexpr int kStageBytes = 4096;   // per warp, on the way out: where the tile's dO was
    static constexpr int kThreads = 384;
    static constexpr int kRegs = 168, kRowRegs = 200, kOtherRegs = 104;   // at launch; then two warpgroups, one
    static_assert(2 * kRowRegs + kOtherRegs <= 3 * kRegs, "shares of the launch's registers");
    static_assert(4 * kStageBytes <= kBytes, "four warps' rows go out through one tile");
    static constexpr int kSmem = 1024 + (4 + kStages) * kBytes + 512;
};

template <int DP>
__global__ void __launch_bounds__(BwdQ<DP>::kThreads, 1)
attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ AttnDev a) {
    using C = BwdQ<DP>;
    extern __shared__ char smem_raw[];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = a.q_heads / a.kv_heads;
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t sq = base, sdo = base + 2 * C::kBytes, sring = base + 4 * C::kBytes;
    const uint32_t bars = sring + C::kStages * C::kBytes;
    const Jobs jobs(bars, a.wait_limit);
    const uint32_t q_full = bars + Jobs::kBytes, q_empty = q_full + 8, do_full = q_full + 16, raw = q_full + 24, taken = q_full + 32,
                   s_full = q_full + 48, s_read = q_full + 64, dp_full = q_full + 80, ds_full = q_full + 96, done = q_full + 112,
                   full = q_full + 128, empty = full + 8 * C::kStages, tmem_slot = empty + 8 * C::kStages;
    // A key tile is used by S and again by dQ, a value tile by dP alone: the first kKeys places of the ring take key
    // tiles, the others value tiles, each in turn.

    let_next_start();
    if (warp == 8) tmem_alloc(tmem_slot, 512);
    if (threadIdx.x == 0) {
        jobs.init(10);
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        mbar_init(do_full, 1);
        mbar_init(raw, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(taken + 8 * i, 4);
            mbar_init(s_full + 8 * i, 1);
            mbar_init(s_read + 8 * i, 4);
            mbar_init(dp_full + 8 * i, 1);
            mbar_init(ds_full + 8 * i, 4);
            mbar_init(done + 8 * i, 1);
        }
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        fence_barrier_init();
    }
    const bool ranked = warp == 10 && is_ranked(a);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    bool ok = true;
    JobWord w;
    w.kind = kJobNone;

    if (warp >= 8) {
        registers_down<C::kOtherRegs>();
        if (warp == 9) {   // -------------------------------------------- loads
            uint32_t n = 0, tiles = 0, seconds = 0, fixed = 0;   // key tiles, jobs, those with two query tiles, tiles with rows of others so far
            for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
                if (w.kind != kJobWork) continue;
                const uint32_t kv_head = w.head / group, row0 = w.block * 2 * kTile;
                const bool two = row0 + kTile < w.len;
                const uint32_t total = w.block * 2 + 1 + (two ? 1 : 0);
                auto rows = [&](const CUtensorMap *map, int mul, uint32_t to, uint32_t bar) {   // Q or dO of both tiles
                    if (lane == 0) {
                        mbar_expect(bar, (two ? 2 : 1) * C::kBytes);
                        for (int t = 0; t < (two ? 2 : 1); ++t)
                            for (int x = 0; x < C::kSub; ++x)
                                tma_load(to + t * C::kBytes + x * (kTile * 128), map, bar, x * 64, int(w.head) * mul, int(w.first + row0 + t * kTile));
                    }
                };
                auto load = [&](bool is_k, uint32_t u) {   // key or value tile u of the job
                    const uint32_t m = n + u, at = is_k ? m % C::kKeys : C::kKeys + m % C::kValues, use = m / (is_k ? C::kKeys : C::kValues);
                    if (use > 0 && !warp_wait(empty + 8 * at, (use - 1) & 1, a.wait_limit)) return false;
                    const bool ragged = is_k && w.len < (u + 1) * kTile;   // a key behind the sequence has dS = 0, times itself in dQ
                    const uint32_t bar = ragged ? raw : full + 8 * at;
                    if (lane == 0) {
                        mbar_expect(bar, C::kBytes);
                        for (int x = 0; x < C::kSub; ++x)
                            tma_load(sring + at * C::kBytes + x * (kTile * 128), is_k ? &mk : &mv, bar, x * 64,
                                     int(kv_head) * (is_k ? a.k_mul : a.v_mul), int(w.first + u * kTile));
                    }
                    if (ragged) {
                        if (!warp_wait(raw, fixed & 1, a.wait_limit)) return false;
                        ++fixed;
                        zero_tile_rows<C::kSub>(sring + at * C::kBytes, w.len - u * kTile);
                        if (lane == 0) mbar_arrive(full + 8 * at);
                    }
                    return true;
                };
                if (tiles > 0 && !(ok = warp_wait(q_empty, (tiles - 1) & 1, a.wait_limit))) break;
                rows(&mq, a.q_mul, sq, q_full);
                if (!(ok = load(true, 0) && load(false, 0) && (total == 1 || load(true, 1)))) break;
                // dO's place has been the last job's way out
                if (tiles > 0 && !(ok = warp_wait(taken, (tiles - 1) & 1, a.wait_limit))) break;
                if (seconds > 0 && !(ok = warp_wait(taken + 8, (seconds - 1) & 1, a.wait_limit))) break;
                rows(&mdo, a.do_mul, sdo, do_full);
                ++tiles;
                seconds += two;
                for (uint32_t u = 1; ok && u < total; ++u) ok = load(false, u) && (u + 1 >= total || load(true, u + 1));
                if (!ok) break;
                n += total;
            }
            // the CTA must not end, nor its memory be given back, before the last loads and releases have arrived
            if (tiles > 0) {
                mbar_wait(q_full, (tiles - 1) & 1, a.wait_limit);
                mbar_wait(do_full, (tiles - 1) & 1, a.wait_limit);
                if (ok) ok = warp_wait(q_empty, (tiles - 1) & 1, a.wait_limit);
            }
            for (uint32_t i = n > C::kKeys ? n - C::kKeys : 0; i < n; ++i) {
                mbar_wait(full + 8 * (i % C::kKeys), (i / C::kKeys) & 1, a.wait_limit);
                if (ok) ok = warp_wait(empty + 8 * (i % C::kKeys), (i / C::kKeys) & 1, a.wait_limit);
            }
            for (uint32_t i = n > C::kValues ? n - C::kValues : 0; i < n; ++i) {
                mbar_wait(full + 8 * (C::kKeys + i % C::kValues), (i / C::kValues) & 1, a.wait_limit);
                if (ok) ok = warp_wait(empty + 8 * (C::kKeys + i % C::kValues), (i / C::kValues) & 1, a.wait_limit);
            }
        } else if (warp == 8) {   // --------------------------------- products
            if (lane == 0) {   // one thread, as in the forward kernel
                const uint32_t id_s = mma_desc(kTile, false), id_o = mma_desc(DP, true);
                uint32_t tiles = 0, c[2] = {0, 0};   // jobs, key tiles of the first and second query tile so far
                Place key, value;
                auto key_of = [&](const Place &p) { return sring + p.at * C::kBytes; };
                auto value_of = [&](const Place &p) { return sring + (C::kKeys + p.at) * C::kBytes; };
                auto wait_key = [&](const Place &p) { return mbar_wait(full + 8 * p.at, p.phase, a.wait_limit); };
                auto scores = [&](int t, const Place &p) {   // S = Q K^T
                    product_rows<DP>(tmem + t * 128, sq + t * C::kBytes, key_of(p), id_s | a.negate);
                    mma_commit(s_full + 8 * t);
                };
                auto d_probs = [&](int t) {                  // dP = dO V^T, over S
                    if (!mbar_wait(s_read + 8 * t, c[t] & 1, a.wait_limit)) return false;
                    tc_fence_after();
                    product_rows<DP>(tmem + t * 128, sdo + t * C::kBytes, value_of(value), id_s);
                    mma_commit(dp_full + 8 * t);
                    return true;
                };
                auto d_query = [&](int t, bool add) {        // dQ += dS K
                    if (!mbar_wait(ds_full + 8 * t, c[t] & 1, a.wait_limit)) return false;
                    tc_fence_after();
                    product_cols<32>(tmem + 256 + t * 128, tmem + t * 128, key_of(key), id_o, add);
                    ++c[t];
                    return true;
                };
                for (uint32_t k = 0; (ok = jobs.get_alone(k, &w)) && w.kind != kJobStop; ++k) {
                    if (w.kind != kJobWork) continue;
                    const bool two = w.block * 2 * kTile + kTile < w.len;
                    const uint32_t nb0 = w.block * 2 + 1, nb = nb0 + (two ? 1 : 0);   // key tiles of the first tile; of both
                    if (!(ok = mbar_wait(q_full, tiles & 1, a.wait_limit) && wait_key(key))) break;
                    tc_fence_after();
                    scores(0, key);
                    if (two) scores(1, key);
                    if (nb == 1) mma_commit(q_empty);
                    if (!(ok = mbar_wait(do_full, tiles & 1, a.wait_limit))) break;
                    ++tiles;
                    for (uint32_t u = 0; u < nb; ++u) {
                        const bool more = u + 1 < nb;
                        Place next = key;
                        next.template next<C::kKeys>();
                        if (!(ok = mbar_wait(full + 8 * (C::kKeys + value.at), value.phase, a.wait_limit))) break;
                        if (u < nb0 && !(ok = d_probs(0))) break;
                        if (two && !(ok = d_probs(1))) break;
                        mma_commit(empty + 8 * (C::kKeys + value.at));
                        value.template next<C::kValues>();
                        if (more && !(ok = wait_key(next))) break;
                        if (u < nb0) {
                            if (!(ok = d_query(0, u > 0))) break;
                            if (u + 1 < nb0) scores(0, next);
                            else mma_commit(done);
                        }
                        if (two) {
                            if (!(ok = d_query(1, u > 0))) break;
                            if (more) scores(1, next);
                            else mma_commit(done + 8);
                        }
                        mma_commit(empty + 8 * key.at);
                        if (u + 2 == nb) mma_commit(q_empty);   // the last use of Q
                        key = next;
                    }
                    if (!ok) break;
                }
            }
        } else if (warp == 10) {   // ------------------------------------ jobs
            ok = jobs.template run<2 * kTile, true, false>(a, ranked, a.q_heads);
        }
    } else {   // ------------------------------------------- a row of a tile
        registers_up<C::kRowRegs>();
        wait_for_previous();   // for the row terms
        const int t = warp >> 2;
        const uint32_t lanes = (warp & 3) << 21, work = tmem + t * 128 + lanes, local = (warp & 3) * 32 + lane;
        const float2 c2 = make_float2(a.exp2_scale, a.exp2_scale);
        uint32_t it = 0, tiles = 0;   // key tiles and jobs of this tile so far
        for (uint32_t k = 0; (ok = jobs.get(k, &w)) && w.kind != kJobStop; ++k) {
            const uint32_t row0 = w.block * 2 * kTile + t * kTile, row = row0 + local;
            if (w.kind == kJobTail) {
                const uint32_t from = w.first + w.block * 2 * kTile, to = min(w.first + w.len, from + 2 * kTile);
                fill_rows(a.d_q, from, to, w.head, a.head_dim, 256);
            }
            if (w.kind != kJobWork) continue;
            if (row0 < w.len) {
                const uint32_t total = w.block * 2 + 1 + t;
                const float2 term = row < w.len ? a.rows[size_t(w.head) * a.n_tokens + w.first + row] : make_float2(0.f, 0.f);
                const float2 l2 = make_float2(term.x, term.x);
                float row_term = term.y;
                float2 left = make_float2(0.f, 0.f);   // sum of this row's dS: what the row term was off by, as P adds up to one
                for (uint32_t u = 0; u < total; ++u, ++it) {
                    if (!(ok = warp_wait(s_full + 8 * t, it & 1, a.wait_limit))) break;
                    tc_fence_after();
                    float2 p[64];
                    {
                        uint32_t r[4][32];
#pragma unroll
                        for (int i = 0; i < 4; ++i) tmem_ld32(r[i], work + 32 * i);
                        tmem_wait_ld();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_read + 8 * t);
#pragma unroll
                        for (int x = 0; x < 64; ++x) {
                            const uint32_t *v = &r[x / 16][2 * (x % 16)];
                            const float2 y = fma2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), c2, l2);
                            p[x] = make_float2(exp2_approx(y.x), exp2_approx(y.y));
                        }
                    }
                    if (!(ok = warp_wait(dp_full + 8 * t, it & 1, a.wait_limit))) break;
                    tc_fence_after();
                    if (total == 1) {   // the row sees this tile alone: its term is exact without the rounded O
                        float exact = 0.f;
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            uint32_t r[32];
                            tmem_ld32(r, work + 32 * h);
                            tmem_wait_ld();
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const uint32_t col = 32 * h + 2 * x;
                                if (col <= local) exact = fmaf(p[16 * h + x].x, __uint_as_float(r[2 * x]), exact);
                                if (col + 1 <= local) exact = fmaf(p[16 * h + x].y, __uint_as_float(r[2 * x + 1]), exact);
                            }
                        }
                        row_term = exact;
                    }
                    const float2 d2 = make_float2(-row_term, -row_term);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t r[32], ds[16];
                        tmem_ld32(r, work + 32 * h);
                        tmem_wait_ld();
                        if (u == total - 1) {   // the diagonal tile: what is hidden may hold anything
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const uint32_t col = 32 * h + 2 * x;
                                float2 y = mul2(p[16 * h + x], add2(make_float2(__uint_as_float(r[2 * x]), __uint_as_float(r[2 * x + 1])), d2));
                                if (col > local) y.x = 0.f;
                                if (col + 1 > local) y.y = 0.f;
                                left = add2(left, y);
                                ds[x] = bf16x2(y.x, y.y);
                            }
                        } else {
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const float2 y = mul2(p[16 * h + x], add2(make_float2(__uint_as_float(r[2 * x]), __uint_as_float(r[2 * x + 1])), d2));
                                left = add2(left, y);
                                ds[x] = bf16x2(y.x, y.y);
                            }
                        }
                        tmem_st16(work + 16 * h, ds);   // over what has been read of dP
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ds_full + 8 * t);
                }
                if (!ok) break;
                // the kernel for dK and dV goes on with the better row term
                if (row < w.len) a.rows[size_t(w.head) * a.n_tokens + w.first + row].y = row_term + (left.x + left.y);
                if (!(ok = warp_wait(done + 8 * t, tiles & 1, a.wait_limit))) break;
                ++tiles;
                tc_fence_after();
                const uint32_t row_w = row - lane;   // the warp's first row
                store_rows<DP, 64>(sdo + t * C::kBytes + (warp & 3) * C::kStageBytes, tmem + 256 + t * 128 + lanes, a.scale, a.d_q,
                                   w.first + row_w, w.head, w.len > row_w ? w.len - row_w : 0u, a.head_dim);
                tc_fence_before();
                fence_async_shared();   // before the next dO lands where the rows went through
                __syncwarp();
                if (lane == 0) mbar_arrive(taken + 8 * t);
            }
        }
    }
    tc_fence_before();
    const bool bad = __syncthreads_or(!ok);
    tc_fence_after();
    if (warp == 8) tmem_free(tmem, 512);
    if (bad) {
        if (w.kind == kJobWork) {   // each warp's own last job
            const uint32_t from = w.first + w.block * 2 * kTile;
            poison_rows(a.d_q, from, min(w.first + w.len, from + 2 * kTile), w.head, a.head_dim);
        }
        if (threadIdx.x == 0) atomicAdd(&g_attn_faults, 1u);
    }
}

}  // namespace
