// Rotary positions on the query and key heads of a pack of tokens (gac_rotary and gac_rotary_on_axes of
// include/gac.h).
//
//   (x, y) -> scale (x cos a - y sin a, x sin a + y cos a),   a = position * freq,   the position that of the pair's axis
//
// Bound by HBM: every element is read once and written once, three flops each.  A CTA takes one token: its threads work
// out the token's sines and cosines (the angle is reduced to one turn in binary64, then sincospi in binary32: exact to
// the last bits at any position, no table in memory) and leave them in shared memory for every head of the token,
// whose first vectors are on their way meanwhile.
// 16384 tokens x 32 heads x 128, bfloat16: 46 to 48 us = 5.6 to 5.8 TB/s (0.86 to 0.90 of a plain copy's rate); 8189 tokens x 14 heads x 128,
// float32, half of the head turned: 22 us = 5.3 TB/s.  The first on three axes, each pair's position read for itself: 45 to
// 49 us.  With 256 threads, 4 tokens to a CTA and the sines made before the loads the first takes 54 us.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "gac.h"
#include "gac_host.h"
#include "rotary.cuh"

namespace {

// Any size, stride and alignment: one pair, or one copied element, at a time.
template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads)
rotary_any_kernel(const __grid_constant__ RotaryDev a) {
    __shared__ float2 wheel[GAC_ROTARY_MAX_DIM / 2];
    const uint32_t t = blockIdx.x;
    fill_wheel<true>(a, wheel, t);
    const uint32_t rest = a.head_dim - 2 * a.pairs, units = a.pairs + rest;
    const uint32_t heads = a.heads[0] + a.heads[1];
    for (uint32_t w = threadIdx.x; w < heads * units; w += kThreads) {
        const uint32_t u = w % units, h0 = w / units;
        const int which = h0 >= a.heads[0];
        const uint32_t h = which ? h0 - a.heads[0] : h0;
        const char *x = a.x[which] + ((long long)t * a.x_token[which] + (long long)h * a.x_head[which]) * (long long)sizeof(T);
        char *y = a.y[which] + ((long long)t * a.y_token[which] + (long long)h * a.y_head[which]) * (long long)sizeof(T);
        if (u < a.pairs) {
            const uint32_t i = HALF ? u : 2 * u, j = HALF ? u + a.pairs : 2 * u + 1;
            const float2 cs = wheel[u];
            const float p = load_el(x + i * sizeof(T), T{}), q = load_el(x + j * sizeof(T), T{});
            store_el(y + i * sizeof(T), p * cs.x - q * cs.y, T{});
            store_el(y + j * sizeof(T), p * cs.y + q * cs.x, T{});
        } else {
            const uint32_t i = a.pairs + u;
            if (x != y) store_el(y + i * sizeof(T), load_el(x + i * sizeof(T), T{}), T{});
        }
    }
}

// A thread keeps one place of the head, N pairs (two vectors) or 2 N copied elements, and walks over the token's heads.
template <typename T, bool HALF, bool AXES>
__global__ void __launch_bounds__(kThreads, 12)
rotary_kernel(const __grid_constant__ RotaryDev a) {
    constexpr int N = 4;
    __shared__ __align__(16) float2 wheel[GAC_ROTARY_MAX_DIM / 2];
    constexpr int kFlight = 2;
    constexpr uint32_t kSize = sizeof(T);
    const uint32_t t = blockIdx.x;
    const uint32_t turned = a.pairs / N, units = turned + (a.head_dim - 2 * a.pairs + 2 * N - 1) / (2 * N);   // places of a head
    const uint32_t u = threadIdx.x % units, step = kThreads / units, heads = a.heads[0] + a.heads[1];
    const bool turn = u < turned;
    // byte offsets of the two vectors in a head
    const uint32_t first = (turn ? (HALF ? u * N : 2 * u * N) : 2 * a.pairs + (u - turned) * 2 * N) * kSize;
    const uint32_t second = first + (turn && HALF ? a.pairs : N) * kSize;
    const bool both = turn || second < a.head_dim * kSize;
    // in place there is nothing to copy
    const bool active = threadIdx.x < step * units && (turn || a.x[0] != a.y[0] || a.x[1] != a.y[1]);
    uint32_t h = active ? threadIdx.x / units : heads;
    Vec<T, N> p[kFlight], q[kFlight];
    char *to[kFlight];   // nullptr: no head
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            to[i] = nullptr;
            if (h >= heads) continue;
            const int which = h >= a.heads[0];
            const uint32_t hh = which ? h - a.heads[0] : h;
            const char *x = a.x[which] + ((long long)t * a.x_token[which] + (long long)hh * a.x_head[which]) * kSize;
            to[i] = a.y[which] + ((long long)t * a.y_token[which] + (long long)hh * a.y_head[which]) * kSize;
            p[i].load(x + first);
            if (both) q[i].load(x + second);
            h += step;
        }
    };
    fetch();   // on its way while the sines are made
    fill_wheel<AXES>(a, wheel, t);
    while (to[0]) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (!to[i]) break;
            if (turn) {
                const float4 *cs = reinterpret_cast<const float4 *>(wheel + u * N);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float4 c = cs[j / 2];   // cosine, sine, cosine, sine
                    if (HALF) {
                        const float x0 = p[i].get(j), x1 = p[i].get(j + 1), y0 = q[i].get(j), y1 = q[i].get(j + 1);
                        p[i].put2(j, x0 * c.x - y0 * c.y, x1 * c.z - y1 * c.w);
                        q[i].put2(j, x0 * c.y + y0 * c.x, x1 * c.w + y1 * c.z);
                    } else {
                        Vec<T, N> &v = j < N / 2 ? p[i] : q[i];
                        const int e = 2 * j - (j < N / 2 ? 0 : N);
                        const float x0 = v.get(e), y0 = v.get(e + 1), x1 = v.get(e + 2), y1 = v.get(e + 3);
                        v.put2(e, x0 * c.x - y0 * c.y, x0 * c.y + y0 * c.x);
                        v.put2(e + 2, x1 * c.z - y1 * c.w, x1 * c.w + y1 * c.z);
                    }
                }
            }
            p[i].store(to[i] + first);
            if (both) q[i].store(to[i] + second);
        }
        fetch();
    }
}

}  // namespace

extern "C" {

int gac_rotary_freqs(double *freqs, uint32_t rot_dim, double base, int scaling, double factor, double trained, double low,
                     double high) {
    if (!freqs) return fail(nullptr, GAC_ERR_INVALID_ARG, "freqs is NULL%s");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > GAC_ROTARY_MAX_DIM)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "rot_dim must be even, 2..%s%lld", "", GAC_ROTARY_MAX_DIM);
    if (!(base > 1.0) || !isfinite(base)) return fail(nullptr, GAC_ERR_INVALID_ARG, "base must be finite and > 1%s");
    if (!(factor >= 1.0) || !isfinite(factor)) return fail(nullptr, GAC_ERR_INVALID_ARG, "factor must be finite and >= 1%s");
    if (scaling < GAC_ROTARY_NONE || scaling > GAC_ROTARY_PARTS) return fail(nullptr, GAC_ERR_INVALID_ARG, "unknown scaling%s");
    if (scaling == GAC_ROTARY_NONE && factor != 1.0)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "a factor needs a scaling%s");
    if (scaling == GAC_ROTARY_BASE && rot_dim == 2)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "scaling the base needs rot_dim > 2%s");
    if (scaling == GAC_ROTARY_PARTS && (!(trained > 0.0) || !isfinite(trained) || !(low >= 0.0) || !(high > low) || !isfinite(high)))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "scaling by parts needs trained > 0 and 0 <= low < high%s");
    const double r = double(rot_dim);
    if (scaling == GAC_ROTARY_BASE) base *= pow(factor, r / (r - 2.0));
    for (uint32_t i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / r);
        if (scaling == GAC_ROTARY_LINEAR) f /= factor;
        if (scaling == GAC_ROTARY_PARTS) {
            const double turns = trained * f / (2.0 * M_PI);
            const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
            f *= keep + (1.0 - keep) / factor;
        }
        freqs[i] = f;
    }
    return GAC_OK;
}

int gac_rotary_on_axes(const gac_rotary_args *args, const gac_rotary_axes *axes, int cuda_device, void *cuda_stream) {
    if (!args) return fail(nullptr, GAC_ERR_INVALID_ARG, "args is NULL%s");
    const gac_rotary_args &a = *args;
    RotaryDev d;
    Rows x[2], y[2];
    const int rc = check_rotary(a, axes, false, d, x, y);
    if (rc != GAC_OK) return rc;
    if (a.n_tokens == 0 || (a.heads[0] == 0 && a.heads[1] == 0)) return GAC_OK;
    Range range("gac_rotary");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool half = a.layout == GAC_ROTARY_HALF, bf16 = a.dtype == GAC_BF16;
    // Vectors of four elements where every vector of every head starts on such a boundary and ends inside its part of the
    // head, single elements otherwise: 16384 tokens x 32 heads x 128 bfloat16 take 46 us and 110 (vectors of eight: 48).
    const bool vectors = vectors_fit(d, 4, bf16 ? 2 : 4);
    void (*fn)(const RotaryDev) = nullptr;
    if (vectors && axes) fn = bf16 ? (half ? rotary_kernel<uint16_t, true, true> : rotary_kernel<uint16_t, false, true>)
                                   : (half ? rotary_kernel<float, true, true> : rotary_kernel<float, false, true>);
    else if (vectors) fn = bf16 ? (half ? rotary_kernel<uint16_t, true, false> : rotary_kernel<uint16_t, false, false>)
                                : (half ? rotary_kernel<float, true, false> : rotary_kernel<float, false, false>);
    else fn = bf16 ? (half ? rotary_any_kernel<uint16_t, true> : rotary_any_kernel<uint16_t, false>)
                   : (half ? rotary_any_kernel<float, true> : rotary_any_kernel<float, false>);
    fn<<<a.n_tokens, kThreads, 0, s>>>(d);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

int gac_rotary(const gac_rotary_args *args, int cuda_device, void *cuda_stream) {
    return gac_rotary_on_axes(args, nullptr, cuda_device, cuda_stream);
}

}  // extern "C"
