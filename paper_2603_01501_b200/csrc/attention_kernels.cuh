// Device code of causal attention over packed sequences for sm_100a.  Included by attention.cu only.
#pragma once

#include <math.h>
#include <stdint.h>

#include "gac.h"
#include "sm100.cuh"

namespace {

constexpr int kTile = 128;                  // rows of a query or key tile: one tcgen05 accumulator
constexpr float kLog2e = 1.4426950408889634f;

// Set by a kernel whose bounded wait ran out; read and cleared by gac_attn_check.
static __device__ int g_attn_fault;

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
    const char *o_in, *do_in;          // backward: for the row terms
    long long do_token, do_head;
    float *lse, *delta;
};

// cu_seqlens entry b, kept in range; entry 0 is taken as 0.
__device__ __forceinline__ uint32_t seq_bound(const AttnDev &a, uint32_t b) {
    if (b == 0) return 0u;
    const int32_t c = __ldg(a.cu + b);
    return c < 0 ? 0u : min(uint32_t(c), a.n_tokens);
}

// Which rows a CTA works on.  Every sequence gets the slots  start/ROWS + b ... : at least as many as it has
// blocks of ROWS rows, found without a prefix sum over the pack (some slots stay empty).  The rows behind the
// last sequence are slot range n_seqs.
struct Slot {
    uint32_t first, len;   // the sequence
    uint32_t row;          // first row of the block within it
    bool tail;
};
template <int ROWS>
__device__ __forceinline__ Slot find_slot(const AttnDev &a, uint32_t slot) {   // whole warps
    uint32_t lo = 0, hi = a.n_seqs;   // the last b in [lo, hi] with start(b) <= slot
    while (hi - lo > 31) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (seq_bound(a, mid) / ROWS + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    const uint32_t b0 = lo + (threadIdx.x & 31);
    const bool here = b0 <= hi && seq_bound(a, b0) / ROWS + b0 <= slot;
    const uint32_t found = __ballot_sync(0xFFFFFFFFu, here);
    const uint32_t b = lo + (found ? 31 - __clz(found) : 0);
    Slot s;
    s.first = seq_bound(a, b);
    s.tail = (b == a.n_seqs);
    const uint32_t end = s.tail ? a.n_tokens : max(s.first, seq_bound(a, b + 1));
    s.len = end - s.first;
    s.row = (slot - (s.first / ROWS + b)) * ROWS;
    return s;
}
inline uint32_t slot_count(uint32_t n_tokens, uint32_t n_seqs, uint32_t rows) { return n_tokens / rows + n_seqs + 1; }

// Writes one bit pattern over `dim` elements of rows [from, to) of one head, by the whole CTA: zero for rows that
// belong to no sequence, NaN where a wait ran out.
constexpr uint32_t kZeroBits = 0u, kNanBits = 0x7FFF7FFFu;
__device__ __forceinline__ void fill_rows(const RowsOut &o, uint32_t from, uint32_t to, uint32_t head, uint32_t dim, uint32_t bits) {
    const uint32_t per = dim / 8, n = (to - from) * per;
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
        char *p = o.p + (long long)(from + i / per) * o.token + (long long)head * o.head + (i % per) * 16;
        *reinterpret_cast<uint4 *>(p) = make_uint4(bits, bits, bits, bits);
    }
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
// Warps: 0-3 and 4-7 the rows of the two tiles, 8 issues the products, 9 the TMA loads.

template <int DP>
struct Fwd {
    static constexpr int kSub = DP / 64;                     // 64-wide blocks of a row
    static constexpr int kBytes = kTile * DP * 2;            // one tile
    static constexpr int kStages = DP == 128 ? 5 : 8;        // key and value tiles in flight
    static constexpr int kThreads = 320;
    static constexpr int kSmem = 1024 + (2 + kStages) * kBytes + 256;
};

template <int DP>
__global__ void __launch_bounds__(Fwd<DP>::kThreads, 1)
attn_forward_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, const __grid_constant__ AttnDev a) {
    using C = Fwd<DP>;
    extern __shared__ char smem_raw[];
    const uint32_t head = blockIdx.x % a.q_heads, kv_head = head / (a.q_heads / a.kv_heads);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Slot s = find_slot<2 * kTile>(a, (gridDim.x - 1 - blockIdx.x) / a.q_heads);   // the longest rows first
    if (s.row >= s.len) return;
    if (s.tail) {
        const uint32_t from = s.first + s.row, to = min(s.first + s.len, from + 2 * kTile);
        fill_rows(a.o, from, to, head, a.head_dim, kZeroBits);
        for (uint32_t t = from + threadIdx.x; t < to; t += blockDim.x) a.lse[size_t(head) * a.n_tokens + t] = -INFINITY;
        return;
    }
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t sq = base, sring = base + 2 * C::kBytes;
    const uint32_t bars = sring + C::kStages * C::kBytes;
    const uint32_t q_full = bars, s_full = bars + 8, p_full = bars + 24, o_full = bars + 40, full = bars + 56,
                   empty = full + 8 * C::kStages, tmem_slot = empty + 8 * C::kStages;
    const bool two = s.row + kTile < s.len;
    const uint32_t nb0 = s.row / kTile + 1, nb = nb0 + (two ? 1 : 0);   // key tiles of the first tile; of both

    if (warp == 8) tmem_alloc(tmem_slot, 512);
    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
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
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    bool ok = true;

    if (warp == 9) {   // ------------------------------------------------ loads
        if (lane == 0) {
            mbar_expect(q_full, (two ? 2 : 1) * C::kBytes);
            for (int t = 0; t < (two ? 2 : 1); ++t)
                for (int x = 0; x < C::kSub; ++x)
                    tma_load(sq + t * C::kBytes + x * (kTile * 128), &mq, q_full, x * 64, int(head) * a.q_mul,
                             int(s.first + s.row + t * kTile));
            uint32_t n = 0;
            for (; n < 2 * nb; ++n) {
                const uint32_t st = n % C::kStages, use = n / C::kStages;
                if (use > 0 && !(ok = mbar_wait(empty + 8 * st, (use - 1) & 1))) break;
                const bool is_k = (n & 1) == 0;
                mbar_expect(full + 8 * st, C::kBytes);
                for (int x = 0; x < C::kSub; ++x)
                    tma_load(sring + st * C::kBytes + x * (kTile * 128), is_k ? &mk : &mv, full + 8 * st, x * 64,
                             int(kv_head) * (is_k ? a.k_mul : a.v_mul), int(s.first + (n / 2) * kTile));
            }
            if (!ok)   // the copies in flight have to land before the memory is given back
                for (uint32_t i = n > C::kStages ? n - C::kStages : 0; i < n; ++i)
                    mbar_wait(full + 8 * (i % C::kStages), (i / C::kStages) & 1);
        }
    } else if (warp == 8) {   // ------------------------------------- products
        const uint32_t id_s = mma_desc(kTile, false) | a.negate, id_o = mma_desc(DP, true);
        auto scores = [&](int t, uint32_t j) {   // S_t = Q_t K_j^T
            const uint32_t n = 2 * j, k = sring + (n % C::kStages) * C::kBytes, q = sq + t * C::kBytes;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    const uint32_t off = (i / 4) * (kTile * 128) + (i % 4) * 32;
                    mma_ss(tmem + t * 128, smem_desc(q + off, 0), smem_desc(k + off, 0), id_s, i > 0);
                }
                mma_commit(s_full + 8 * t);
            }
        };
        auto values = [&](int t, uint32_t j) {   // O_t += P_t V_j
            const uint32_t n = 2 * j + 1, v = sring + (n % C::kStages) * C::kBytes;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < kTile / 16; ++i)
                    mma_ts(tmem + 256 + t * 128, tmem + t * 128 + i * 8, smem_desc(v + i * 2048, kTile * 128), id_o, j > 0 || i > 0);
                mma_commit(o_full + 8 * t);
            }
        };
        auto wait_tile = [&](uint32_t n) { return warp_wait(full + 8 * (n % C::kStages), (n / C::kStages) & 1); };
        auto release = [&](uint32_t n) {
            if (lane == 0 && n + C::kStages < 2 * nb) mma_commit(empty + 8 * (n % C::kStages));   // somebody waits for it
        };
        ok = warp_wait(q_full, 0) && wait_tile(0);
        if (ok) {
            tc_fence_after();
            scores(0, 0);
            if (two) scores(1, 0);
            release(0);
        }
        for (uint32_t j = 0; ok && j < nb; ++j) {
            if (!(ok = wait_tile(2 * j + 1))) break;
            if (j + 1 < nb && !(ok = wait_tile(2 * j + 2))) break;
            if (j == nb - 1 && s.len < (j + 1) * kTile) {
                // rows of V behind the sequence belong to others: their P is zero, but zero times a NaN is not
                const uint32_t from = s.len - j * kTile;
                const uint32_t v = sring + ((2 * j + 1) % C::kStages) * C::kBytes;
                for (int x = 0; x < C::kSub; ++x)
                    for (uint32_t i = from * 8 + lane; i < kTile * 8; i += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v + x * (kTile * 128) + i * 16), "r"(0) : "memory");
                fence_async_shared();
                __syncwarp();
            }
            if (j < nb0) {
                if (!(ok = warp_wait(p_full, j & 1))) break;
                tc_fence_after();
                values(0, j);
                if (j + 1 < nb0) scores(0, j + 1);
            }
            if (two) {
                if (!(ok = warp_wait(p_full + 8, j & 1))) break;
                tc_fence_after();
                values(1, j);
                release(2 * j + 1);
                if (j + 1 < nb) {
                    scores(1, j + 1);
                    release(2 * j + 2);
                }
            } else {
                release(2 * j + 1);
                if (j + 1 < nb) release(2 * j + 2);
            }
        }
    } else if (warp < 4 || two) {   // -------------------------- a row of a tile
        const int t = warp >> 2;
        const uint32_t my_blocks = nb0 + t, lanes = (warp & 3) << 21;   // tensor memory lane 32 (warp & 3)
        const uint32_t ts = tmem + t * 128 + lanes, to = tmem + 256 + t * 128 + lanes;
        const uint32_t local = (warp & 3) * 32 + lane;
        const float c = a.exp2_scale;
        float m = -INFINITY;
        float2 sum = make_float2(0.f, 0.f);
        for (uint32_t j = 0; j < my_blocks; ++j) {
            if (!(ok = warp_wait(s_full + 8 * t, j & 1))) break;
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
            for (int i = 0; i < 128; ++i) mx[i % 4] = fmaxf(mx[i % 4], __uint_as_float(r[i / 32][i % 32]));
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
            if (j == 0) m = top;
            else if (__any_sync(0xFFFFFFFFu, (top - m) * c > 8.0f)) {
                if (!(ok = warp_wait(o_full + 8 * t, (j - 1) & 1))) break;
                tc_fence_after();
                const float next = fmaxf(m, top), f = exp2_approx((m - next) * c);
                const float2 f2 = make_float2(f, f);
                sum = mul2(sum, f2);
                m = next;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    uint32_t w[32];
                    tmem_ld32(w, to + 32 * i);
                    tmem_wait_ld();
#pragma unroll
                    for (int u = 0; u < 32; ++u) w[u] = __float_as_uint(__uint_as_float(w[u]) * f);
                    tmem_st32(to + 32 * i, w);
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
        if (ok) ok = warp_wait(o_full + 8 * t, (my_blocks - 1) & 1);
        if (ok) {
            tc_fence_after();
            const float total = sum.x + sum.y, inv = 1.0f / total;
            const uint32_t row = s.row + t * kTile + local;
            const bool mine = row < s.len;
            char *out = a.o.p + (long long)(s.first + row) * a.o.token + (long long)head * a.o.head;
            if (mine)
                a.lse[size_t(head) * a.n_tokens + s.first + row] = m * fabsf(a.scale) + logf(total);
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                uint32_t w[32];
                tmem_ld32(w, to + 32 * i);
                tmem_wait_ld();
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float *f = reinterpret_cast<const float *>(w + 8 * u);
                    const uint4 v = make_uint4(bf16x2(f[0] * inv, f[1] * inv), bf16x2(f[2] * inv, f[3] * inv),
                                               bf16x2(f[4] * inv, f[5] * inv), bf16x2(f[6] * inv, f[7] * inv));
                    if (mine && 32 * i + 8 * u < int(a.head_dim)) *reinterpret_cast<uint4 *>(out + (32 * i + 8 * u) * 2) = v;
                }
            }
        }
    }
    tc_fence_before();
    const bool bad = __syncthreads_or(!ok);
    tc_fence_after();
    if (warp == 8) tmem_free(tmem, 512);
    if (bad) {
        const uint32_t from = s.first + s.row, to = min(s.first + s.len, from + 2 * kTile);
        fill_rows(a.o, from, to, head, a.head_dim, kNanBits);
        for (uint32_t t = from + threadIdx.x; t < to; t += blockDim.x)
            a.lse[size_t(head) * a.n_tokens + t] = __int_as_float(0x7FFFFFFF);
        if (threadIdx.x == 0) g_attn_fault = 1;
    }
}

}  // namespace
