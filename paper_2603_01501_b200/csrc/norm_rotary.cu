// Norms of query and key heads with their rotation in the same pass, and its way back (gac_norm_rotary,
// gac_norm_rotary_backward of include/gac.h).
//
//   r = 1 / sqrt(mean_d x_d^2 + eps),   y = R (x r w),   w = offset + weight,   R: the turn, with its scale
//   a = R^T dy,   dw = sum a x r,   b = a w,   dx = r (b - x r^2 mean_d(b_d x_d))
//
// r is made again on the way back: x has to be read there in any case.  All arithmetic is binary32, results are rounded
// once.  The lanes that share a head have one place of it each, and the place's sines and weights in registers for as many
// heads of their token as they take, so that a head costs little more than its loads, a product with r and the turn.  The shares of dw
// that CTAs keep in registers are added up by a second launch, in binary64 and a fixed order, so two calls give the same bits.
//
// Bound by HBM and by instructions: 16384 tokens x 32 heads x 128, bfloat16, take 50 us (5.4 TB/s, 0.83 of a plain copy's rate; the
// turn alone, gac_rotary, 45), 65 % of the issue slots used; 12291 tokens x 14 heads 21 us and 31 back, where three tensors
// pass (4.7 TB/s in the kernel's 28).  With a token to a CTA and weights and sines in shared memory the same took 70 us, and 90 in
// both directions: 400 instructions for four heads of a warp instead of 240, many of them divisions and 64-bit products.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "gac.h"
#include "gac_host.h"
#include "rotary.cuh"
#include "sm100.cuh"

namespace {

constexpr uint32_t kMaxDim = 1024, kMaxVectorDim = 256;
constexpr int kForwardCtas = 5, kBackCtas = 4;   // of an SM
constexpr uint32_t kShares = 148 * kBackCtas;    // most CTAs of the way back for one kind of heads, each with a share of the weights' gradient
constexpr uint32_t kFew = 1u << 18;              // elements of all heads: about one place for each thread of all SMs
constexpr int kRing = 3;                         // heads that a thread has loads of on their way

struct NormDev {
    const char *w[2];                 // nullptr: ones, without offset
    int w_bf16;
    float eps, offset, inv_dim;
    uint32_t group;                   // lanes of a head: a power of two
    uint32_t ctas_q;                  // CTAs; on the way back those that take query heads, while the others take key heads
    uint32_t split[2];                // a token's heads are dealt out to so many groups of lanes
    long long x_token[2], x_head[2], y_token[2], y_head[2];   // RotaryDev's strides in bytes
    long long x_step[2], y_step[2], v_step[2];                // and from a head to the next one of the same lanes
    // the way back: RotaryDev's x is d_y, its y is d_x
    const char *v[2];                 // the heads that went in
    long long v_token[2], v_head[2];  // bytes
    float *shares;                    // [CTAs][head_dim]: of query heads, then of key heads
};

__device__ __forceinline__ float weight_at(const NormDev &n, int which, uint32_t i) {
    if (!n.w[which]) return 1.0f;
    return n.offset + (n.w_bf16 ? load_el(n.w[which] + i * 2, uint16_t{}) : load_el(n.w[which] + i * 4, float{}));
}
__device__ __forceinline__ float add_lanes(float x, uint32_t group) {
#pragma unroll
    for (uint32_t o = 1; o < 32; o *= 2)
        if (o < group) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// A thread's place in a head: N elements from `first`, N from `second`, so that the lanes of a head read and write one behind the
// other.  The two are the elements of N pairs, or N / 2 pairs each, or not turned.
struct Part {
    uint32_t u, first, second;
    bool here, turn, both;
};
template <int N>
__device__ __forceinline__ Part part_of(const RotaryDev &a, const NormDev &n) {
    const uint32_t turned = a.pairs / N, rest = (a.head_dim - 2 * a.pairs) / N, places = turned + (rest + 1) / 2;
    Part p;
    p.u = threadIdx.x & (n.group - 1);
    p.here = p.u < places;
    p.turn = p.u < turned;
    p.first = p.turn ? p.u * N : 2 * a.pairs + (p.u - turned) * N;
    p.second = p.first + (p.turn ? a.pairs : (rest + 1) / 2 * N);
    p.both = p.here && (p.turn || p.second < a.head_dim);
    return p;
}
// N elements of a place, two to a number, out of 8 or 16 bytes of shared memory, and into as many of global memory.
template <typename T, int N>
__device__ __forceinline__ void take(uint32_t from, float2 *v) {
    Vec<T, N> p;
    constexpr int kWords = Vec<T, N>::kWords;
    if (kWords == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[kWords - 2]), "=r"(p.w[kWords - 1]) : "r"(from) : "memory");
    else
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(p.w[0]), "=r"(p.w[1]) : "r"(from) : "memory");
#pragma unroll
    for (int j = 0; j < N; j += 2) v[j / 2] = make_float2(p.get(j), p.get(j + 1));
}
template <typename T, int N>
__device__ __forceinline__ void put(char *to, const float2 *v) {
    Vec<T, N> p;
#pragma unroll
    for (int j = 0; j < N; j += 2) p.put2(j, v[j / 2].x, v[j / 2].y);
    p.store(to);
}
// (x, y) -> (a x - b y, c x + d y) on a place's N pairs; `minus_b` has the sign already.  v: two elements each, as they lie in the head.
template <int N, bool HALF>
__device__ __forceinline__ void turn(float2 (&v)[N], const float2 *a, const float2 *minus_b, const float2 *c, const float2 *d) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if (HALF) {
            const float2 x = v[i], y = v[N / 2 + i];
            v[i] = fma2(x, a[i], mul2(y, minus_b[i]));
            v[N / 2 + i] = fma2(x, c[i], mul2(y, d[i]));
        } else {
            const float2 p = v[2 * i], q = v[2 * i + 1];
            v[2 * i] = make_float2(fmaf(p.x, a[i].x, p.y * minus_b[i].x), fmaf(p.x, c[i].x, p.y * d[i].x));
            v[2 * i + 1] = make_float2(fmaf(q.x, a[i].y, q.y * minus_b[i].y), fmaf(q.x, c[i].y, q.y * d[i].y));
        }
    }
}

// The lanes that share a head keep to one token, with its sines in registers, and go through every `split`-th of its query heads and
// then of its key heads; on the way back the first ctas_q CTAs take query heads and the others key heads, for there is no room for both
// weights' gradients.  What a thread will need next is on its way into its own places of a ring in shared memory.  No two threads
// share anything but the sums over a head, and on the way back the last sum over the CTA.
template <typename T, int N, bool HALF, bool BACK>
__global__ void __launch_bounds__(kThreads, BACK ? kBackCtas : kForwardCtas)
norm_rotary_kernel(const __grid_constant__ RotaryDev a, const __grid_constant__ NormDev n) {
    constexpr int kBytes = N * int(sizeof(T)), kLoads = BACK ? 4 : 2, kStage = kLoads * kThreads * kBytes;
    extern __shared__ __align__(16) char dynamic[];
    __shared__ long long steps[GAC_ROTARY_MAX_DIM / 2];      // 2^64 turns per position, of each pair
    __shared__ float2 weights[2 * kMaxVectorDim];            // of each kind of heads: the places' 2 N elements
    if (BACK) let_next_start();
    const uint32_t ring = smem_addr(dynamic) + threadIdx.x * kBytes;
    const uint32_t groups = kThreads / n.group;
    const bool keys = BACK && blockIdx.x >= n.ctas_q;
    const uint32_t cta = keys ? blockIdx.x - n.ctas_q : blockIdx.x, ctas = keys ? gridDim.x - n.ctas_q : n.ctas_q;
    const int kind0 = BACK ? keys : a.heads[0] == 0, kind1 = BACK ? keys : a.heads[1] != 0;
    const uint32_t split = n.split[kind0];
    const uint32_t units = a.n_tokens * split, all = ctas * groups, unit0 = cta * groups + threadIdx.x / n.group;
    const uint32_t turns = (units + all - 1) / all;   // of units, as many for every group of lanes
    const Part at = part_of<N>(a, n);
    const uint32_t apart = (at.second - at.first) * uint32_t(sizeof(T));
    auto rounds_of = [&](int kind) { return (a.heads[kind] + split - 1) / split; };

    auto fetch = [&](const char *row, uint32_t to) {
        auto copy = [&](uint32_t dst, const char *src) {
            if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
        };
        if (at.here) copy(to, row);
        if (at.both) copy(to + kThreads * kBytes, row + apart);
    };
    // what comes in next: a round of a kind of heads of a unit
    uint32_t f_turn = 0, f_left = 0, f_head = 0;
    int f_kind = kind0;
    bool f_live = false;
    const char *f_x = nullptr, *f_v = nullptr;
    auto issue = [&](uint32_t slot) {
        if (f_turn < turns) {
            if (f_left == 0) {
                const uint32_t unit = unit0 + f_turn * all;
                const long long t = unit / split;
                f_left = rounds_of(f_kind);
                f_live = unit < units;
                f_head = unit % split;
                f_x = a.x[f_kind] + t * n.x_token[f_kind] + (long long)f_head * n.x_head[f_kind] + at.first * sizeof(T);
                if (BACK) f_v = n.v[f_kind] + t * n.v_token[f_kind] + (long long)f_head * n.v_head[f_kind] + at.first * sizeof(T);
            }
            if (f_live && f_head < a.heads[f_kind]) {
                const uint32_t to = ring + slot * kStage;
                fetch(f_x, to);
                if (BACK) fetch(f_v, to + 2 * kThreads * kBytes);
            }
            f_head += split;
            f_x += n.x_step[f_kind];
            if (BACK) f_v += n.v_step[f_kind];
            if (--f_left == 0) {
                f_turn += f_kind == kind1;
                f_kind = f_kind == kind1 ? kind0 : kind1;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // what is not there of a head stays zero in the ring
    for (int i = 0; i < kRing * kLoads; ++i)
        if (!(i % 2 ? at.both : at.here))
            for (int w = 0; w < kBytes / 4; ++w) asm volatile("st.shared.u32 [%0], %1;" ::"r"(ring + i * kThreads * kBytes + w * 4), "r"(0) : "memory");
#pragma unroll
    for (int i = 0; i < kRing; ++i) issue(i);

    for (uint32_t i = threadIdx.x; i < a.pairs; i += kThreads) steps[i] = __double2ll_rn((a.turns[i] - rint(a.turns[i])) * 18446744073709551616.0);
    for (uint32_t k = threadIdx.x / n.group; k < 2; k += groups)
        for (int i = 0; i < N; ++i) {
            const bool there = i < N / 2 ? at.here : at.both;
            const uint32_t e = i < N / 2 ? at.first + 2 * i : at.second + 2 * i - N;
            weights[(k * n.group + at.u) * N + i] = there ? make_float2(weight_at(n, k, e), weight_at(n, k, e + 1)) : make_float2(0.f, 0.f);
        }
    __syncthreads();
    float2 w[N];
    auto weigh = [&](int kind) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = weights[(kind * n.group + at.u) * N + i];
    };
    if (BACK) weigh(kind0);

    float2 dw[BACK ? N : 1] = {};
    uint32_t slot = 0;
    for (uint32_t step = 0; step < turns; ++step) {
        const uint32_t unit = unit0 + step * all, t = unit / split;
        const bool live = unit < units;
        // cosines and sines of the place's pairs; what is not turned stays as it is.  The angle is a whole number of 2^-64 turns,
        // so whole turns fall away by themselves
        float2 cosines[N / 2], sines[N / 2];
        const int place = live && at.turn && !a.positions ? place_in_sequence(a.cu, a.n_seqs, t) : 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            float2 cs[2] = {make_float2(1.f, 0.f), make_float2(1.f, 0.f)};
            if (live && at.turn)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t k = 2 * i + j, pair = HALF ? at.u * N + k : (k < N / 2 ? 0 : a.pairs / 2 - N / 2) + at.u * (N / 2) + k;
                    // unsigned, for it is meant to overflow
                    const long long angle = (long long)((unsigned long long)steps[pair] * (unsigned long long)(long long)(a.positions ? position_on_axis(a, pair, t) : place));
                    float s, c;
                    sincospif(__ll2float_rn(angle) * 1.0842021724855044e-19f, &s, &c);   // 2^-63: halves of a turn, 24 bits of any angle
                    cs[j] = make_float2(c * a.scale, s * a.scale);
                }
            cosines[i] = make_float2(cs[0].x, cs[1].x);
            sines[i] = make_float2(cs[0].y, cs[1].y);
        }
        for (int kind = kind0; kind <= kind1; ++kind) {
            // x -> a x - b y, y -> c x + d y, forward with the weights in them
            float2 ma[BACK ? 1 : N / 2], mb[BACK ? 1 : N / 2], mc[BACK ? 1 : N / 2], md[BACK ? 1 : N / 2];
            if constexpr (!BACK) {
                weigh(kind);
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const float2 wx = HALF ? w[i] : make_float2(w[2 * i].x, w[2 * i + 1].x), wy = HALF ? w[N / 2 + i] : make_float2(w[2 * i].y, w[2 * i + 1].y);
                    ma[i] = mul2(cosines[i], wx);
                    mb[i] = mul2(make_float2(-sines[i].x, -sines[i].y), wy);
                    mc[i] = mul2(sines[i], wx);
                    md[i] = mul2(cosines[i], wy);
                }
            }
            const uint32_t heads = a.heads[kind], rounds = rounds_of(kind);
            uint32_t h = unit % split;
            char *to = a.y[kind] + (long long)t * n.y_token[kind] + (long long)h * n.y_head[kind] + at.first * sizeof(T);
            for (uint32_t round = 0; round < rounds; ++round, h += split, to += n.y_step[kind]) {
                float2 v[N], squares = make_float2(0.f, 0.f);
                const uint32_t from = ring + slot * kStage;
                const bool here = live && h < heads;
                asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
                if constexpr (!BACK) {
                    take<T, N>(from, v);
                    take<T, N>(from + kThreads * kBytes, v + N / 2);
                    issue(slot);
#pragma unroll
                    for (int j = 0; j < N; ++j) squares = fma2(v[j], v[j], squares);
                    const float r = rsqrtf(fmaf(add_lanes(squares.x + squares.y, n.group), n.inv_dim, n.eps));
#pragma unroll
                    for (int j = 0; j < N; ++j) v[j] = mul2(v[j], make_float2(r, r));
                    turn<N, HALF>(v, ma, mb, mc, md);
                } else {
                    float2 b[N], bw[N], dot = squares, minus[N / 2];
                    take<T, N>(from, b);
                    take<T, N>(from + kThreads * kBytes, b + N / 2);
                    take<T, N>(from + 2 * kThreads * kBytes, v);
                    take<T, N>(from + 3 * kThreads * kBytes, v + N / 2);
                    issue(slot);
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) minus[i] = make_float2(-sines[i].x, -sines[i].y);
                    turn<N, HALF>(b, cosines, sines, minus, cosines);   // by the negative angle
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        bw[j] = mul2(b[j], w[j]);
                        squares = fma2(v[j], v[j], squares);
                        dot = fma2(bw[j], v[j], dot);
                    }
                    const float r = rsqrtf(fmaf(add_lanes(squares.x + squares.y, n.group), n.inv_dim, n.eps));
                    const float c = -(add_lanes(dot.x + dot.y, n.group) * n.inv_dim * r * r);
                    const float2 rr = make_float2(r, r);
                    if (here)
#pragma unroll
                        for (int j = 0; j < N; ++j) dw[j] = fma2(b[j], mul2(v[j], rr), dw[j]);
#pragma unroll
                    for (int j = 0; j < N; ++j) v[j] = mul2(rr, fma2(v[j], make_float2(c, c), bw[j]));
                }
                slot = slot + 1 == kRing ? 0 : slot + 1;
                if (here && at.here) put<T, N>(to, v);
                if (here && at.both) put<T, N>(to + apart, v + N / 2);
            }
        }
    }
    if constexpr (BACK) {
        // the CTA's share: the threads of one place in their order
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        float *sums = reinterpret_cast<float *>(dynamic);   // 2 N of a thread: no more than the ring
        static_assert(2 * N * sizeof(float) <= size_t(kRing) * kLoads * kBytes, "fits the ring");
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) sums[i * kThreads + threadIdx.x] = i & 1 ? dw[i / 2].y : dw[i / 2].x;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * N * n.group; i += kThreads) {   // groups of lanes are powers of two, as the threads are
            const uint32_t j = i / n.group;
            const float *from = sums + j * kThreads + at.u;
            float s = 0.f;
            for (uint32_t m = 0; m < groups; ++m) s += from[m * n.group];
            if (j < N ? at.here : at.both) n.shares[size_t(blockIdx.x) * a.head_dim + (j < N ? at.first + j : at.second + j - N)] = s;
        }
    }
}

// Any size, stride and alignment: a warp to a head, a pair or an element that is not turned to a lane.
template <typename T, bool HALF, bool BACK>
__global__ void __launch_bounds__(kThreads)
norm_rotary_any_kernel(const __grid_constant__ RotaryDev a, const __grid_constant__ NormDev n) {
    __shared__ float2 wheel[GAC_ROTARY_MAX_DIM / 2];
    extern __shared__ float dw[];   // the way back: [warps][queries, keys][head_dim], every element one lane's
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, heads = a.heads[0] + a.heads[1];
    const uint32_t units = a.head_dim - a.pairs;
    constexpr long long kSize = sizeof(T);
    if (BACK)
        for (uint32_t i = threadIdx.x; i < kThreads / 32 * 2 * a.head_dim; i += kThreads) dw[i] = 0.f;
    for (uint32_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
        __syncthreads();   // all are done with the wheel
        fill_wheel<true>(a, wheel, t);
        for (uint32_t h0 = warp; h0 < heads; h0 += kThreads / 32) {
            const int which = h0 >= a.heads[0];
            const uint32_t h = which ? h0 - a.heads[0] : h0;
            const char *in = a.x[which] + ((long long)t * a.x_token[which] + (long long)h * a.x_head[which]) * kSize;
            const char *v = BACK ? n.v[which] + (long long)t * n.v_token[which] + (long long)h * n.v_head[which] : in;
            char *y = a.y[which] + ((long long)t * a.y_token[which] + (long long)h * a.y_head[which]) * kSize;
            // The unit's elements i and, if it is a pair, j; what comes in, turned back on the way back; and the weights
            auto unit = [&](uint32_t u, uint32_t &i, uint32_t &j, float &p, float &q) {
                const bool pair = u < a.pairs;
                i = !pair ? a.pairs + u : HALF ? u : 2 * u;
                j = !pair ? i : HALF ? u + a.pairs : 2 * u + 1;
                p = load_el(in + i * kSize, T{});
                q = pair ? load_el(in + j * kSize, T{}) : 0.f;
                if (BACK && pair) {
                    const float2 cs = wheel[u];
                    const float x0 = p, y0 = q;
                    p = x0 * cs.x + y0 * cs.y;
                    q = y0 * cs.x - x0 * cs.y;
                }
                return pair;
            };
            float squares = 0.f, dot = 0.f;
            for (uint32_t u = lane; u < units; u += 32) {
                uint32_t i, j;
                float p, q;
                const bool pair = unit(u, i, j, p, q);
                const float vi = BACK ? load_el(v + i * kSize, T{}) : p, vj = !pair ? 0.f : BACK ? load_el(v + j * kSize, T{}) : q;
                squares = fmaf(vi, vi, fmaf(vj, vj, squares));
                if (BACK) dot = fmaf(p * weight_at(n, which, i), vi, fmaf(q * weight_at(n, which, j), vj, dot));
            }
            const float r = rsqrtf(fmaf(add_lanes(squares, 32), n.inv_dim, n.eps));
            const float c = BACK ? add_lanes(dot, 32) * n.inv_dim * r * r : 0.f;
            for (uint32_t u = lane; u < units; u += 32) {
                uint32_t i, j;
                float p, q;
                const bool pair = unit(u, i, j, p, q);
                const float wi = weight_at(n, which, i), wj = weight_at(n, which, j);
                if (BACK) {
                    float *acc = dw + (warp * 2 + which) * a.head_dim;
                    const float vi = load_el(v + i * kSize, T{}), vj = pair ? load_el(v + j * kSize, T{}) : 0.f;
                    acc[i] += p * (vi * r);
                    if (pair) acc[j] += q * (vj * r);
                    p = r * fmaf(-vi, c, p * wi);
                    q = r * fmaf(-vj, c, q * wj);
                } else {
                    p = p * r * wi;
                    q = q * r * wj;
                    if (pair) {
                        const float2 cs = wheel[u];
                        const float x0 = p, y0 = q;
                        p = x0 * cs.x - y0 * cs.y;
                        q = x0 * cs.y + y0 * cs.x;
                    }
                }
                store_el(y + i * kSize, p, T{});
                if (pair) store_el(y + j * kSize, q, T{});
            }
        }
    }
    if (!BACK) return;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * a.head_dim; i += kThreads) {
        float s = 0.f;
        for (uint32_t m = 0; m < kThreads / 32; ++m) s += dw[m * 2 * a.head_dim + i];
        n.shares[(size_t(i >= a.head_dim) * gridDim.x + blockIdx.x) * a.head_dim + i % a.head_dim] = s;
    }
}

// d_weight[which][i] = sum of the shares, eight columns to a CTA: 128 threads to a column, each with a few loads in flight.
constexpr uint32_t kColumns = 8, kColumnThreads = 128;
struct WeightsDev {
    const float *shares;
    char *d_w[2];
    int w_bf16;
    uint32_t first[2], count[2], head_dim;   // shares of each kind of heads; columns
};
__global__ void __launch_bounds__(kColumns *kColumnThreads) norm_weights_kernel(const __grid_constant__ WeightsDev a) {
    __shared__ double sums[32][kColumns];
    const uint32_t c = threadIdx.x % kColumns, row = threadIdx.x / kColumns, tiles = (a.head_dim + kColumns - 1) / kColumns;
    const int which = blockIdx.x >= tiles;
    const uint32_t col = (blockIdx.x - which * tiles) * kColumns + c, count = a.count[which];
    wait_for_previous();
    double s = 0.0;
    if (col < a.head_dim) {
        const float *from = a.shares + size_t(a.first[which]) * a.head_dim + col;
#pragma unroll 4
        for (uint32_t i = row; i < count; i += kColumnThreads) s += double(__ldcg(from + size_t(i) * a.head_dim));
    }
#pragma unroll
    for (int o = kColumns; o < 32; o *= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);   // the warp's four rows
    if (threadIdx.x % 32 < kColumns) sums[threadIdx.x / 32][c] = s;
    __syncthreads();
    if (row != 0 || col >= a.head_dim || !a.d_w[which]) return;
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][c];
    if (a.w_bf16) store_el(a.d_w[which] + col * 2, float(s), uint16_t{});
    else store_el(a.d_w[which] + col * 4, float(s), float{});
}

uint32_t share_count(const gac_rotary_args &a) { return std::min(a.n_tokens, kShares); }

// Checks the weights and fills `n`; `d` has been checked.
int check_norm(const gac_rotary_args &a, const gac_norm &norm, const Rows (&y)[2], NormDev &n) {
    if (a.inverse) return fail(nullptr, GAC_ERR_INVALID_ARG, "inverse must be 0 with norms%s");
    if (norm.weight_dtype != GAC_F32 && norm.weight_dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "weights are float32 or bfloat16%s");
    if (norm.reserved != 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "reserved must be 0%s");
    if (!(norm.eps > 0.0) || !isfinite(norm.eps) || !(float(norm.eps) > 0.f) || !isfinite(float(norm.eps)))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "eps must be positive and finite in float32%s");
    if (!isfinite(norm.offset)) return fail(nullptr, GAC_ERR_INVALID_ARG, "offset must be finite%s");
    if (a.head_dim < 1) return fail(nullptr, GAC_ERR_INVALID_ARG, "head_dim must be at least 1%s");
    const uint64_t size = norm.weight_dtype == GAC_BF16 ? 2 : 4;
    n.w_bf16 = norm.weight_dtype == GAC_BF16;
    n.eps = float(norm.eps);
    n.offset = float(norm.offset);
    n.inv_dim = 1.0f / float(a.head_dim);
    for (int w = 0; w < 2; ++w) {
        n.w[w] = static_cast<const char *>(norm.weight[w]);
        if (reinterpret_cast<uint64_t>(n.w[w]) % size) return fail(nullptr, GAC_ERR_INVALID_ARG, "a weight is misaligned%s");
        if (!n.w[w] || a.n_tokens == 0) continue;
        const Rows r = rows_of(n.w[w], 0, 0, 1, 1, a.head_dim, size);
        for (int i = 0; i < 2; ++i)
            if (a.heads[i] && share(y[i], r)) return fail(nullptr, GAC_ERR_INVALID_ARG, "output heads overlap a weight%s");
    }
    return GAC_OK;
}

// How a launch of the vector kernel is laid out, N elements to a vector.
struct Layout {
    uint32_t grid, smem;
};
Layout lay_out(const RotaryDev &d, NormDev &n, uint32_t elements, uint32_t size, bool back) {
    n.group = 1;
    while (n.group * 2 * elements < d.head_dim) n.group *= 2;
    const uint32_t groups = kThreads / n.group, most = 148 * (back ? kBackCtas : kForwardCtas);
    // Into how many groups of lanes a token's heads are split: what a group has to do is to be least, `turns` tokens with their sines,
    // which take about as long as kSines heads; and no more CTAs than it takes for all to have the same number of tokens.
    const uint32_t kSines = back ? 4 : 8;
    auto share_out = [&](uint32_t ctas, uint32_t heads0, uint32_t heads1, uint32_t *split) {
        uint64_t least = ~uint64_t(0), most_turns = 1;
        for (uint32_t s = 1; s <= groups && s < 2 * std::max(heads0, heads1); s *= 2) {
            const uint64_t turns = (uint64_t(d.n_tokens) * s + uint64_t(ctas) * groups - 1) / (uint64_t(ctas) * groups);
            const uint64_t work = turns * ((heads0 + s - 1) / s + (heads1 + s - 1) / s + kSines);
            if (work >= least) continue;
            least = work;
            most_turns = turns;
            *split = s;
        }
        return uint32_t(((uint64_t(d.n_tokens) * *split + most_turns - 1) / most_turns + groups - 1) / groups);
    };
    uint32_t grid = 0;
    if (back) {
        // CTAs are shared out to the kinds by what a token of each takes
        const uint32_t cost[2] = {d.heads[0] ? d.heads[0] + kSines : 0, d.heads[1] ? d.heads[1] + kSines : 0};
        for (int w = 0; w < 2; ++w) {
            n.split[w] = 1;
            if (d.heads[w]) grid += share_out(std::max(1u, most * cost[w] / (cost[0] + cost[1])), d.heads[w], 0, &n.split[w]);
            if (w == 0) n.ctas_q = grid;
        }
    } else {
        n.ctas_q = grid = share_out(most, d.heads[0], d.heads[1], &n.split[0]);
        n.split[1] = n.split[0];
    }
    for (int w = 0; w < 2; ++w) {
        n.x_token[w] = d.x_token[w] * size;
        n.x_head[w] = d.x_head[w] * size;
        n.y_token[w] = d.y_token[w] * size;
        n.y_head[w] = d.y_head[w] * size;
        n.x_step[w] = n.x_head[w] * n.split[w];
        n.y_step[w] = n.y_head[w] * n.split[w];
        n.v_step[w] = back ? n.v_head[w] * n.split[w] : 0;
    }
    return Layout{grid, uint32_t(kRing) * (back ? 4 : 2) * kThreads * elements * size};
}
template <bool BACK>
void (*vector_kernel(uint32_t elements, bool bf16, bool half))(const RotaryDev, const NormDev) {
    if (!bf16) return half ? norm_rotary_kernel<float, 4, true, BACK> : norm_rotary_kernel<float, 4, false, BACK>;
    if (elements == 8) return half ? norm_rotary_kernel<uint16_t, 8, true, BACK> : norm_rotary_kernel<uint16_t, 8, false, BACK>;
    return half ? norm_rotary_kernel<uint16_t, 4, true, BACK> : norm_rotary_kernel<uint16_t, 4, false, BACK>;
}

}  // namespace

extern "C" {

int gac_norm_rotary(const gac_rotary_args *args, const gac_rotary_axes *axes, const gac_norm *norm, int cuda_device, void *cuda_stream) {
    if (!args || !norm) return fail(nullptr, GAC_ERR_INVALID_ARG, "args or norm is NULL%s");
    const gac_rotary_args &a = *args;
    RotaryDev d;
    NormDev n;
    Rows x[2], y[2];
    int rc = check_rotary(a, axes, true, d, x, y);
    if (rc == GAC_OK) rc = check_norm(a, *norm, y, n);
    if (rc != GAC_OK) return rc;
    if (a.n_tokens == 0 || (a.heads[0] == 0 && a.heads[1] == 0)) return GAC_OK;
    Range range("gac_norm_rotary");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool half = a.layout == GAC_ROTARY_HALF, bf16 = a.dtype == GAC_BF16;
    // Vectors of 16 bytes, or of four bfloat16, where every vector of every head starts on such a boundary; else single elements.
    uint32_t elements = 0;
    // A few tokens take the shorter ones: twice the lanes to a head, each with half as many sines to make.
    const bool few = uint64_t(a.n_tokens) * (a.heads[0] + a.heads[1]) * a.head_dim < uint64_t(kFew);
    if (a.head_dim <= kMaxVectorDim) elements = bf16 && !few && vectors_fit(d, 8, 2) ? 8 : vectors_fit(d, 4, bf16 ? 2 : 4) ? 4 : 0;
    if (elements) {
        const Layout how = lay_out(d, n, elements, bf16 ? 2 : 4, false);
        vector_kernel<false>(elements, bf16, half)<<<how.grid, kThreads, how.smem, s>>>(d, n);
    } else {
        void (*fn)(const RotaryDev, const NormDev) =
            bf16 ? (half ? norm_rotary_any_kernel<uint16_t, true, false> : norm_rotary_any_kernel<uint16_t, false, false>)
                 : (half ? norm_rotary_any_kernel<float, true, false> : norm_rotary_any_kernel<float, false, false>);
        fn<<<a.n_tokens, kThreads, 0, s>>>(d, n);
    }
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

size_t gac_norm_rotary_workspace(const gac_rotary_args *args) {
    if (!args || args->head_dim > kMaxDim) return 0;
    return size_t(share_count(*args)) * 2 * args->head_dim * sizeof(float);
}

int gac_norm_rotary_backward(const gac_rotary_args *args, const gac_rotary_axes *axes, const gac_norm *norm, const gac_norm_grad *grad,
                             int cuda_device, void *cuda_stream) {
    if (!args || !norm || !grad) return fail(nullptr, GAC_ERR_INVALID_ARG, "args, norm or grad is NULL%s");
    const gac_rotary_args &a = *args;
    RotaryDev d;
    NormDev n;
    Rows x[2], y[2];
    int rc = check_rotary(a, axes, true, d, x, y);
    if (rc == GAC_OK) rc = check_norm(a, *norm, y, n);
    if (rc != GAC_OK) return rc;
    const uint64_t size = a.dtype == GAC_BF16 ? 2 : 4, w_size = n.w_bf16 ? 2 : 4;
    const bool heads = a.n_tokens != 0 && (a.heads[0] != 0 || a.heads[1] != 0);
    const size_t need = gac_norm_rotary_workspace(args);
    if (heads && (!grad->workspace || reinterpret_cast<uint64_t>(grad->workspace) % 16 || grad->workspace_bytes < need))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace is missing, misaligned or too small%s");
    auto aligned = [&](uint32_t elements) {   // the forward call's heads too
        for (int w = 0; w < 2; ++w)
            if (a.heads[w] && (reinterpret_cast<uint64_t>(grad->x[w].p) % (elements * size) || grad->x[w].token % elements || grad->x[w].head % elements))
                return false;
        return a.head_dim <= kMaxVectorDim && vectors_fit(d, elements, size);
    };
    // What is written shares no memory with anything else (d_y and d_x have been checked: apart, or one and the same).
    Rows in[6], out[3];
    int ins = 0, outs = 0;
    auto refuse = [](const Rows &r, const Rows *with, int count) {
        for (int i = 0; i < count; ++i)
            if (share(r, with[i])) return true;
        return false;
    };
    if (heads) out[outs++] = rows_of(grad->workspace, 0, 0, 1, 1, need, 1);
    for (int w = 0; w < 2; ++w) {
        if (grad->d_weight[w]) {
            if (reinterpret_cast<uint64_t>(grad->d_weight[w]) % w_size) return fail(nullptr, GAC_ERR_INVALID_ARG, "a weight's gradient is misaligned%s");
            out[outs] = rows_of(grad->d_weight[w], 0, 0, 1, 1, a.head_dim, w_size);
            if (refuse(out[outs], out, outs)) return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace and the weights' gradients overlap%s");
            ++outs;
        }
        if (norm->weight[w]) in[ins++] = rows_of(norm->weight[w], 0, 0, 1, 1, a.head_dim, w_size);
        n.v[w] = static_cast<const char *>(grad->x[w].p);
        n.v_token[w] = grad->x[w].token * int64_t(size);
        n.v_head[w] = grad->x[w].head * int64_t(size);
        if (!heads || a.heads[w] == 0) continue;
        const uint64_t p = reinterpret_cast<uint64_t>(n.v[w]);
        const int64_t most = int64_t(1) << 40;
        if (!p || p % size || grad->x[w].token < 0 || grad->x[w].head < 0 || grad->x[w].token > most || grad->x[w].head > most)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "the heads of the forward call are NULL or misaligned, or their strides out of range%s");
        in[ins++] = rows_of(n.v[w], grad->x[w].token, grad->x[w].head, a.n_tokens, a.heads[w], a.head_dim, size);
    }
    for (int w = 0; w < 2; ++w) {
        if (!heads || a.heads[w] == 0) continue;
        if (refuse(y[w], in, ins)) return fail(nullptr, GAC_ERR_INVALID_ARG, "a gradient of the heads overlaps an input%s");
        if (refuse(y[w], out, outs) || refuse(x[w], out, outs))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace or a weight's gradient overlaps the heads' gradients%s");
    }
    for (int i = 0; i < outs; ++i)
        if (refuse(out[i], in, ins)) return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace or a weight's gradient overlaps an input%s");
    n.shares = static_cast<float *>(grad->workspace);
    Range range("gac_norm_rotary_backward");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool half = a.layout == GAC_ROTARY_HALF, bf16 = a.dtype == GAC_BF16;
    WeightsDev wd = {};
    if (heads) {
        const uint32_t elements = bf16 && aligned(8) ? 8 : aligned(4) ? 4 : 0;
        if (elements) {
            const Layout how = lay_out(d, n, elements, size, true);
            wd.first[1] = wd.count[0] = n.ctas_q;
            wd.count[1] = how.grid - n.ctas_q;
            vector_kernel<true>(elements, bf16, half)<<<how.grid, kThreads, how.smem, s>>>(d, n);
        } else {
            void (*fn)(const RotaryDev, const NormDev) =
                bf16 ? (half ? norm_rotary_any_kernel<uint16_t, true, true> : norm_rotary_any_kernel<uint16_t, false, true>)
                     : (half ? norm_rotary_any_kernel<float, true, true> : norm_rotary_any_kernel<float, false, true>);
            wd.first[1] = wd.count[0] = wd.count[1] = share_count(a);
            fn<<<share_count(a), kThreads, kThreads / 32 * 2 * a.head_dim * sizeof(float), s>>>(d, n);
        }
        GAC_CUDA(nullptr, cudaGetLastError());
    }
    if (grad->d_weight[0] || grad->d_weight[1]) {
        wd.shares = n.shares;
        wd.w_bf16 = n.w_bf16;
        wd.head_dim = a.head_dim;
        for (int w = 0; w < 2; ++w) wd.d_w[w] = static_cast<char *>(grad->d_weight[w]);
        cudaLaunchConfig_t how = {};
        how.gridDim = dim3(2 * ((a.head_dim + kColumns - 1) / kColumns));
        how.blockDim = dim3(kColumns * kColumnThreads);
        how.stream = s;
        cudaLaunchAttribute attr[1];   // set up while the kernel before ends
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = heads ? 1 : 0;
        how.attrs = attr;
        how.numAttrs = 1;
        GAC_CUDA(nullptr, cudaLaunchKernelEx(&how, norm_weights_kernel, wd));
    }
    return GAC_OK;
}

}  // extern "C"
