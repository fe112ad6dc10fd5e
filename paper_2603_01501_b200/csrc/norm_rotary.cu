// Norms of query and key heads with their rotation in the same pass, and its way back (gac_norm_rotary,
// gac_norm_rotary_backward of include/gac.h).
//
//   r = 1 / sqrt(mean_d x_d^2 + eps),   y = R (x r w),   w = offset + weight,   R: the turn, with its scale
//   a = R^T dy,   dw = sum a x r,   b = a w,   dx = r (b - x r^2 mean_d(b_d x_d))
//
// r is made again on the way back: x has to be read there in any case.  All arithmetic is binary32, results are rounded
// once.  A thread keeps one place of the head (four pairs, or eight elements that are not turned) and the lanes of a head
// add up their squares; a CTA's threads walk over the heads of a token, with the token's sines and both weights in shared
// memory.  On the way back a CTA takes every gridDim-th token and keeps its share of dw in registers; a second launch adds up the
// shares, in binary64 and a fixed order, so two calls give the same bits.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "gac.h"
#include "gac_host.h"
#include "rotary.cuh"

namespace {

constexpr uint32_t kMaxDim = 1024, kMaxVectorDim = 256;
constexpr uint32_t kShares = 148 * 8;   // most CTAs of the way back, each with a share of the weights' gradients

struct NormDev {
    const char *w[2];                 // nullptr: ones, without offset
    int w_bf16;
    float eps, offset, inv_dim;
    uint32_t group;                   // lanes of a head: a power of two
    // the way back: RotaryDev's x is d_y, its y is d_x
    const char *v[2];                 // the heads that went in
    long long v_token[2], v_head[2];
    float *shares;                    // [CTAs][queries, keys][head_dim]
};

__device__ __forceinline__ float weight_at(const NormDev &n, int which, uint32_t i) {
    if (!n.w[which]) return 1.0f;
    return n.offset + (n.w_bf16 ? load_el(n.w[which] + i * 2, uint16_t{}) : load_el(n.w[which] + i * 4, float{}));
}
__device__ __forceinline__ void fill_weights(const RotaryDev &a, const NormDev &n, float *w) {
    for (uint32_t i = threadIdx.x; i < 2 * a.head_dim; i += kThreads) w[i] = weight_at(n, i >= a.head_dim, i >= a.head_dim ? i - a.head_dim : i);
}
__device__ __forceinline__ float add_lanes(float x, uint32_t group) {
    for (uint32_t o = group / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// A thread's place in a head: elements 0..3 start at `first`, 4..7 at `second`.
struct Part {
    uint32_t u, first, second;
    bool here, turn, both;
};
template <bool HALF>
__device__ __forceinline__ Part part_of(const RotaryDev &a, const NormDev &n) {
    const uint32_t turned = a.pairs / 4, units = turned + (a.head_dim - 2 * a.pairs + 7) / 8;
    Part p;
    p.u = threadIdx.x & (n.group - 1);
    p.here = p.u < units;
    p.turn = p.u < turned;
    p.first = p.turn ? (HALF ? p.u * 4 : p.u * 8) : 2 * a.pairs + (p.u - turned) * 8;
    p.second = p.first + (p.turn && HALF ? a.pairs : 4);
    p.both = p.here && (p.turn || p.second < a.head_dim);
    return p;
}
template <typename T>
struct Eight {
    Vec<T, 4> p, q;
    __device__ __forceinline__ void load(const char *row, const Part &at) {
        if (at.here) p.load(row + at.first * sizeof(T));
        if (at.both) q.load(row + at.second * sizeof(T));
    }
    __device__ __forceinline__ void get(float (&v)[8], const Part &at) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = at.here ? p.get(j) : 0.f;
            v[4 + j] = at.both ? q.get(j) : 0.f;
        }
    }
    __device__ __forceinline__ void put(const float (&v)[8], char *row, const Part &at) {
        p.put2(0, v[0], v[1]);
        p.put2(2, v[2], v[3]);
        q.put2(0, v[4], v[5]);
        q.put2(2, v[6], v[7]);
        if (at.here) p.store(row + at.first * sizeof(T));
        if (at.both) q.store(row + at.second * sizeof(T));
    }
};
__device__ __forceinline__ void eight_floats(float (&v)[8], const float *row, const Part &at) {
    const float4 x = *reinterpret_cast<const float4 *>(row + (at.here ? at.first : 0));
    const float4 y = *reinterpret_cast<const float4 *>(row + (at.both ? at.second : 0));
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
}
// The place's four pairs by their angles, or by the negative ones.
template <bool HALF, bool BACK>
__device__ __forceinline__ void turn(float (&v)[8], const float2 *wheel, const Part &at) {
    if (!at.turn) return;
    const float4 *cs = reinterpret_cast<const float4 *>(wheel + at.u * 4);
#pragma unroll
    for (int m = 0; m < 4; m += 2) {
        const float4 c = cs[m / 2];   // cosine, sine, cosine, sine
        const int i0 = HALF ? m : 2 * m, j0 = HALF ? m + 4 : 2 * m + 1, i1 = HALF ? m + 1 : 2 * m + 2, j1 = HALF ? m + 5 : 2 * m + 3;
        const float s0 = BACK ? -c.y : c.y, s1 = BACK ? -c.w : c.w;
        const float x0 = v[i0], y0 = v[j0], x1 = v[i1], y1 = v[j1];
        v[i0] = x0 * c.x - y0 * s0;
        v[j0] = x0 * s0 + y0 * c.x;
        v[i1] = x1 * c.z - y1 * s1;
        v[j1] = x1 * s1 + y1 * c.z;
    }
}

template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads, 8)
norm_rotary_kernel(const __grid_constant__ RotaryDev a, const __grid_constant__ NormDev n) {
    constexpr int kFlight = 2;
    __shared__ __align__(16) float2 wheel[GAC_ROTARY_MAX_DIM / 2];
    __shared__ __align__(16) float weights[2 * kMaxVectorDim];
    const uint32_t t = blockIdx.x, step = kThreads / n.group, heads = a.heads[0] + a.heads[1];
    const Part at = part_of<HALF>(a, n);
    uint32_t h = threadIdx.x / n.group;
    Eight<T> x[kFlight];
    char *to[kFlight];   // nullptr: no head
    const float *w[kFlight];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < kFlight; ++i, h += step) {
            to[i] = nullptr;
            w[i] = weights;
            if (h >= heads) continue;
            const int which = h >= a.heads[0];
            const uint32_t hh = which ? h - a.heads[0] : h;
            to[i] = a.y[which] + ((long long)t * a.y_token[which] + (long long)hh * a.y_head[which]) * (long long)sizeof(T);
            w[i] = weights + which * a.head_dim;
            x[i].load(a.x[which] + ((long long)t * a.x_token[which] + (long long)hh * a.x_head[which]) * (long long)sizeof(T), at);
        }
    };
    fetch();   // on its way while the sines are made
    fill_weights(a, n, weights);
    fill_wheel<true>(a, wheel, t);
    for (uint32_t done = 0; done < heads; done += kFlight * step) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            float v[8], k[8], sum = 0.f;
            x[i].get(v, at);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
            const float r = rsqrtf(fmaf(add_lanes(sum, n.group), n.inv_dim, n.eps));
            if (!to[i]) continue;
            eight_floats(k, w[i], at);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * r * k[j];
            turn<HALF, false>(v, wheel, at);
            x[i].put(v, to[i], at);
        }
        fetch();
    }
}

template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads, 8)
norm_rotary_back_kernel(const __grid_constant__ RotaryDev a, const __grid_constant__ NormDev n) {
    __shared__ __align__(16) float2 wheels[2][GAC_ROTARY_MAX_DIM / 2];
    __shared__ __align__(16) float weights[2 * kMaxVectorDim];
    __shared__ float sums[kThreads * 16];
    const uint32_t step = kThreads / n.group, heads = a.heads[0] + a.heads[1], mine = threadIdx.x / n.group;
    const Part at = part_of<HALF>(a, n);
    float dw[2][8] = {};
    fill_weights(a, n, weights);
    uint32_t turn_of = 0;
    for (uint32_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x, turn_of ^= 1) {
        float2 *wheel = wheels[turn_of];
        Eight<T> g, x;
        char *to;
        int which;
        uint32_t h = mine;
        auto fetch = [&]() {
            to = nullptr;
            which = h >= a.heads[0];
            if (h < heads) {
                const uint32_t hh = which ? h - a.heads[0] : h;
                to = a.y[which] + ((long long)t * a.y_token[which] + (long long)hh * a.y_head[which]) * (long long)sizeof(T);
                g.load(a.x[which] + ((long long)t * a.x_token[which] + (long long)hh * a.x_head[which]) * (long long)sizeof(T), at);
                x.load(n.v[which] + ((long long)t * n.v_token[which] + (long long)hh * n.v_head[which]) * (long long)sizeof(T), at);
            }
            h += step;
        };
        fetch();
        fill_wheel<true>(a, wheel, t);   // the other wheel is done with once all have come here
        for (uint32_t done = 0; done < heads; done += step) {
            float b[8], v[8], k[8], squares = 0.f, dot = 0.f;
            g.get(b, at);
            x.get(v, at);
            turn<HALF, true>(b, wheel, at);
            eight_floats(k, weights + (to && which ? a.head_dim : 0), at);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                squares = fmaf(v[j], v[j], squares);
                dot = fmaf(b[j] * k[j], v[j], dot);
            }
            const float r = rsqrtf(fmaf(add_lanes(squares, n.group), n.inv_dim, n.eps));
            const float c = add_lanes(dot, n.group) * n.inv_dim * r * r;
            if (to) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float share = b[j] * (v[j] * r);
                    if (which) dw[1][j] += share;
                    else dw[0][j] += share;
                    b[j] = r * fmaf(-v[j], c, b[j] * k[j]);
                }
                g.put(b, to, at);
            }
            fetch();
        }
    }
    // the CTA's share: the threads of one place in their order
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[i * kThreads + threadIdx.x] = dw[i / 8][i % 8];
    __syncthreads();
    if (threadIdx.x < n.group && at.here) {
        float *to = n.shares + size_t(blockIdx.x) * 2 * a.head_dim;
        for (int i = 0; i < 16; ++i) {
            float s = 0.f;
            for (uint32_t m = 0; m < step; ++m) s += sums[i * kThreads + m * n.group + threadIdx.x];
            const int j = i % 8;
            if (j < 4 || at.both) to[(i / 8) * a.head_dim + (j < 4 ? at.first + j : at.second + j - 4)] = s;
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
            const char *v = BACK ? n.v[which] + ((long long)t * n.v_token[which] + (long long)h * n.v_head[which]) * kSize : in;
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
        n.shares[size_t(blockIdx.x) * 2 * a.head_dim + i] = s;
    }
}

// d_weight[which][i] = sum of the shares, 32 columns to a CTA.
struct WeightsDev {
    const float *shares;
    char *d_w[2];
    int w_bf16;
    uint32_t n, head_dim;   // shares, columns
};
__global__ void __launch_bounds__(1024) norm_weights_kernel(const __grid_constant__ WeightsDev a) {
    __shared__ double sums[32][33];
    const uint32_t c = threadIdx.x % 32, row = threadIdx.x / 32, col = blockIdx.x * 32 + c;
    double s = 0.0;
    if (col < 2 * a.head_dim)
        for (uint32_t i = row; i < a.n; i += 32) s += double(a.shares[size_t(i) * 2 * a.head_dim + col]);
    sums[row][c] = s;
    __syncthreads();
    if (row != 0 || col >= 2 * a.head_dim) return;
    for (uint32_t i = 1; i < 32; ++i) s += sums[i][c];
    const int which = col >= a.head_dim;
    const uint32_t i = which ? col - a.head_dim : col;
    if (!a.d_w[which]) return;
    if (a.w_bf16) store_el(a.d_w[which] + i * 2, float(s), uint16_t{});
    else store_el(a.d_w[which] + i * 4, float(s), float{});
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
    n.group = 1;
    while (n.group * 8 < a.head_dim) n.group *= 2;
    return GAC_OK;
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
    void (*fn)(const RotaryDev, const NormDev) = nullptr;
    if (a.head_dim <= kMaxVectorDim && vectors_fit(d, 4, bf16 ? 2 : 4))
        fn = bf16 ? (half ? norm_rotary_kernel<uint16_t, true> : norm_rotary_kernel<uint16_t, false>)
                  : (half ? norm_rotary_kernel<float, true> : norm_rotary_kernel<float, false>);
    else
        fn = bf16 ? (half ? norm_rotary_any_kernel<uint16_t, true, false> : norm_rotary_any_kernel<uint16_t, false, false>)
                  : (half ? norm_rotary_any_kernel<float, true, false> : norm_rotary_any_kernel<float, false, false>);
    fn<<<a.n_tokens, kThreads, 0, s>>>(d, n);
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
    bool vectors = heads && a.head_dim <= kMaxVectorDim && vectors_fit(d, 4, size);
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
        n.v_token[w] = grad->x[w].token;
        n.v_head[w] = grad->x[w].head;
        if (!heads || a.heads[w] == 0) continue;
        const uint64_t p = reinterpret_cast<uint64_t>(n.v[w]);
        const int64_t most = int64_t(1) << 40;
        if (!p || p % size || n.v_token[w] < 0 || n.v_head[w] < 0 || n.v_token[w] > most || n.v_head[w] > most)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "the heads of the forward call are NULL or misaligned, or their strides out of range%s");
        vectors = vectors && p % (4 * size) == 0 && n.v_token[w] % 4 == 0 && n.v_head[w] % 4 == 0;
        in[ins++] = rows_of(n.v[w], n.v_token[w], n.v_head[w], a.n_tokens, a.heads[w], a.head_dim, size);
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
    const uint32_t shares = heads ? share_count(a) : 0;
    if (heads) {
        void (*fn)(const RotaryDev, const NormDev) = nullptr;
        if (vectors)
            fn = bf16 ? (half ? norm_rotary_back_kernel<uint16_t, true> : norm_rotary_back_kernel<uint16_t, false>)
                      : (half ? norm_rotary_back_kernel<float, true> : norm_rotary_back_kernel<float, false>);
        else
            fn = bf16 ? (half ? norm_rotary_any_kernel<uint16_t, true, true> : norm_rotary_any_kernel<uint16_t, false, true>)
                      : (half ? norm_rotary_any_kernel<float, true, true> : norm_rotary_any_kernel<float, false, true>);
        fn<<<shares, kThreads, vectors ? 0 : kThreads / 32 * 2 * a.head_dim * sizeof(float), s>>>(d, n);
        GAC_CUDA(nullptr, cudaGetLastError());
    }
    if (grad->d_weight[0] || grad->d_weight[1]) {
        WeightsDev wd{n.shares, {static_cast<char *>(grad->d_weight[0]), static_cast<char *>(grad->d_weight[1])}, n.w_bf16, shares, a.head_dim};
        norm_weights_kernel<<<(2 * a.head_dim + 31) / 32, 1024, 0, s>>>(wd);
        GAC_CUDA(nullptr, cudaGetLastError());
    }
    return GAC_OK;
}

}  // extern "C"
