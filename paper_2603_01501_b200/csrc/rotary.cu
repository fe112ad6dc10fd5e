// Rotary positions on the query and key heads of a pack of tokens (gac_rotary of include/gac.h).
//
//   (x, y) -> scale (x cos a - y sin a, x sin a + y cos a),   a = position * freq
//
// Bound by HBM: every element is read once and written once, three flops each.  A CTA takes one token: its threads work
// out the token's sines and cosines (the angle is reduced to one turn in binary64, then sincospi in binary32: exact to
// the last bits at any position, no table in memory) and leave them in shared memory for every head of the token,
// whose first vectors are on their way meanwhile.
// 16384 tokens x 32 heads x 128, bfloat16: 46 to 48 us = 5.6 to 5.8 TB/s (0.86 to 0.90 of a plain copy's rate); 8189 tokens x 14 heads x 128,
// float32, half of the head turned: 22 us = 5.3 TB/s.  With 256 threads, 4 tokens to a CTA and the sines made before
// the loads the first takes 54 us.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <cstddef>

#include "gac.h"
#include "gac_host.h"
#include "overlap.h"

namespace {

constexpr int kThreads = 128;

struct RotaryDev {
    const char *x[2];
    char *y[2];
    long long x_token[2], x_head[2], y_token[2], y_head[2];
    uint32_t heads[2];
    uint32_t n_tokens, n_seqs, head_dim, pairs;
    const int32_t *positions, *cu;
    float scale;
    int inverse;
    double turns[GAC_ROTARY_MAX_DIM / 2];   // turns per position of each pair
};

__device__ __forceinline__ float load_el(const char *p, float) { return *reinterpret_cast<const float *>(p); }
__device__ __forceinline__ float load_el(const char *p, uint16_t) {
    return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t *>(p)) << 16);
}
__device__ __forceinline__ void store_el(char *p, float v, float) { *reinterpret_cast<float *>(p) = v; }
__device__ __forceinline__ void store_el(char *p, float v, uint16_t) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.0f), "f"(v));
    *reinterpret_cast<uint16_t *>(p) = uint16_t(r & 0xFFFFu);
}

// Place of token t in its sequence; tokens behind the last sequence are at 0.  The bisection is the one that the attention
// kernels read the entries by, so that entries out of order mean the same sequences here and there.
__device__ int place_in_sequence(const int32_t *cu, uint32_t n_seqs, uint32_t t) {
    uint32_t lo = 0, hi = n_seqs, first = 0;   // the last b with cu[b] <= t, cu[0] taken as 0; where it starts
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2, cut = uint32_t(max(cu[mid], 0));
        if (cut <= t) {
            lo = mid;
            first = max(first, cut);
        } else {
            hi = mid - 1;
        }
    }
    return lo == n_seqs ? 0 : int(t - first);
}

// Cosine and sine, already scaled, of every pair of the CTA's token.
__device__ __forceinline__ void fill_wheel(const RotaryDev &a, float2 *wheel, uint32_t t) {
    for (uint32_t i = threadIdx.x; i < a.pairs; i += kThreads) {
        const int pos = a.positions ? a.positions[t] : place_in_sequence(a.cu, a.n_seqs, t);
        const double turns = double(pos) * a.turns[i];
        float s, c;
        sincospif(2.0f * float(turns - rint(turns)), &s, &c);
        wheel[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
    }
    __syncthreads();
}

// Any size, stride and alignment: one pair, or one copied element, at a time.
template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads)
rotary_any_kernel(const __grid_constant__ RotaryDev a) {
    __shared__ float2 wheel[GAC_ROTARY_MAX_DIM / 2];
    const uint32_t t = blockIdx.x;
    fill_wheel(a, wheel, t);
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

// N consecutive elements as they lie in memory.
template <typename T, int N>
struct Vec {
    static constexpr int kWords = N * int(sizeof(T)) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char *p) {
        if (kWords == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            w[0] = v.x; w[1] = v.y; w[kWords - 2] = v.z; w[kWords - 1] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x; w[1] = v.y;
        }
    }
    __device__ __forceinline__ void store(char *p) const {
        if (kWords == 4) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[kWords - 2], w[kWords - 1]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
    __device__ __forceinline__ float get(int i) const {
        if (sizeof(T) == 4) return __uint_as_float(w[i]);
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void put2(int i, float a, float b) {   // elements i and i + 1, i even
        if (sizeof(T) == 4) {
            w[i] = __float_as_uint(a);
            w[i + 1] = __float_as_uint(b);
        } else {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i / 2]) : "f"(b), "f"(a));
        }
    }
};

// A thread keeps one place of the head, N pairs (two vectors) or 2 N copied elements, and walks over the token's heads.
template <typename T, bool HALF>
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
    fill_wheel(a, wheel, t);
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

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

Rows rows_of(const void *p, int64_t token, int64_t head, uint64_t nt, uint64_t nh, uint64_t dim, uint64_t size) {
    return Rows{reinterpret_cast<uint64_t>(p), uint64_t(token) * size, uint64_t(head) * size, nt, nh, dim * size};
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

int gac_rotary(const gac_rotary_args *args, int cuda_device, void *cuda_stream) {
    if (!args) return fail(nullptr, GAC_ERR_INVALID_ARG, "args is NULL%s");
    const gac_rotary_args &a = *args;
    if (a.dtype != GAC_F32 && a.dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "heads are float32 or bfloat16%s");
    if (a.layout != GAC_ROTARY_HALF && a.layout != GAC_ROTARY_INTERLEAVED) return fail(nullptr, GAC_ERR_INVALID_ARG, "unknown layout%s");
    if ((a.inverse != 0 && a.inverse != 1) || a.reserved != 0)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "inverse must be 0 or 1, reserved 0%s");
    if (a.rot_dim < 2 || a.rot_dim % 2 || a.rot_dim > a.head_dim || a.rot_dim > GAC_ROTARY_MAX_DIM)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "rot_dim must be even, at least 2, at most head_dim and %s%lld", "", GAC_ROTARY_MAX_DIM);
    if (a.head_dim > 1024 || a.heads[0] > 4096 || a.heads[1] > 4096 || a.n_tokens > (1u << 30) || a.n_seqs > (1u << 30))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "head_dim, heads or n_tokens out of range%s");
    if (!a.freqs) return fail(nullptr, GAC_ERR_INVALID_ARG, "freqs is NULL%s");
    if (!isfinite(a.scale)) return fail(nullptr, GAC_ERR_INVALID_ARG, "scale must be finite%s");
    const uint64_t size = a.dtype == GAC_BF16 ? 2 : 4;
    RotaryDev d;
    Rows x[2], y[2];
    int both = 0;
    for (int w = 0; w < 2; ++w) {
        const gac_rotary_heads &h = a.qk[w];
        d.heads[w] = a.heads[w];
        d.x[w] = a.heads[w] ? static_cast<const char *>(h.x) : nullptr;
        d.y[w] = a.heads[w] ? static_cast<char *>(h.y) : nullptr;
        d.x_token[w] = h.x_token;
        d.x_head[w] = h.x_head;
        d.y_token[w] = h.y_token;
        d.y_head[w] = h.y_head;
        if (a.heads[w] == 0 || a.n_tokens == 0) continue;
        const uint64_t xb = reinterpret_cast<uint64_t>(h.x), yb = reinterpret_cast<uint64_t>(h.y);
        if (!xb || !yb || xb % size || yb % size)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "heads have a NULL or misaligned pointer%s");
        const int64_t most = int64_t(1) << 40;
        if (h.x_token < 0 || h.x_head < 0 || h.x_token > most || h.x_head > most || h.y_token < 0 || h.y_head < 0 || h.y_token > most || h.y_head > most)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "strides must be 0..2^40 elements%s");
        // every output element has a place of its own
        const int64_t lesser = std::min(h.y_token, h.y_head), larger = std::max(h.y_token, h.y_head);
        const bool token_less = h.y_token <= h.y_head;
        const uint64_t n_lesser = token_less ? a.n_tokens : a.heads[w], n_larger = token_less ? a.heads[w] : a.n_tokens;
        if ((n_lesser > 1 && lesser < int64_t(a.head_dim)) ||
            (n_larger > 1 && uint64_t(larger) < (n_lesser - 1) * uint64_t(n_lesser > 1 ? lesser : 0) + a.head_dim))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "output heads overlap one another%s");
        x[w] = rows_of(h.x, h.x_token, h.x_head, a.n_tokens, a.heads[w], a.head_dim, size);
        y[w] = rows_of(h.y, h.y_token, h.y_head, a.n_tokens, a.heads[w], a.head_dim, size);
        ++both;
        if (h.x == h.y) {
            if (h.x_token != h.y_token || h.x_head != h.y_head)
                return fail(nullptr, GAC_ERR_INVALID_ARG, "in place needs the same strides%s");
        } else {
            if (x[w].p < y[w].end() && y[w].p < x[w].end())
                return fail(nullptr, GAC_ERR_INVALID_ARG, "input and output heads overlap without being in place%s");
        }
    }
    // views of one fused tensor lie between each other's heads; what one of the two writes must not be what the other
    // reads or writes
    if (both == 2 && (share(y[0], y[1]) || share(y[0], x[1]) || share(y[1], x[0])))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "output heads overlap the heads of the other input or output%s");
    if (a.n_tokens == 0 || (a.heads[0] == 0 && a.heads[1] == 0)) return GAC_OK;
    if (!a.positions && (!a.cu_seqlens || reinterpret_cast<uint64_t>(a.cu_seqlens) % 4))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "positions or cu_seqlens must be given, 4-byte aligned%s");
    if (reinterpret_cast<uint64_t>(a.positions) % 4) return fail(nullptr, GAC_ERR_INVALID_ARG, "positions must be 4-byte aligned%s");
    d.n_tokens = a.n_tokens;
    d.n_seqs = a.n_seqs;
    d.head_dim = a.head_dim;
    d.pairs = a.rot_dim / 2;
    d.positions = a.positions;
    d.cu = a.cu_seqlens;
    d.scale = float(a.scale);
    d.inverse = a.inverse;
    for (uint32_t i = 0; i < d.pairs; ++i) {
        if (!isfinite(a.freqs[i])) return fail(nullptr, GAC_ERR_INVALID_ARG, "frequency %s%lld is not finite", "", i);
        d.turns[i] = a.freqs[i] / (2.0 * M_PI);
    }
    Range range("gac_rotary");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool half = a.layout == GAC_ROTARY_HALF, bf16 = a.dtype == GAC_BF16;
    // Vectors of four elements where every vector of every head starts on such a boundary and ends inside its part of the
    // head, single elements otherwise: 16384 tokens x 32 heads x 128 bfloat16 take 46 us and 110 (vectors of eight: 48).
    auto fits = [&](uint32_t n) {   // n elements
        const uint64_t bytes = n * size;
        if (d.pairs % n || a.head_dim % n) return false;
        for (int w = 0; w < 2; ++w)
            if (d.heads[w] && (reinterpret_cast<uint64_t>(d.x[w]) % bytes || reinterpret_cast<uint64_t>(d.y[w]) % bytes || d.x_token[w] % n ||
                               d.x_head[w] % n || d.y_token[w] % n || d.y_head[w] % n))
                return false;
        return true;
    };
    const bool vectors = fits(4);
    void (*fn)(const RotaryDev) = nullptr;
    if (vectors) fn = bf16 ? (half ? rotary_kernel<uint16_t, true> : rotary_kernel<uint16_t, false>)
                           : (half ? rotary_kernel<float, true> : rotary_kernel<float, false>);
    else fn = bf16 ? (half ? rotary_any_kernel<uint16_t, true> : rotary_any_kernel<uint16_t, false>)
                   : (half ? rotary_any_kernel<float, true> : rotary_any_kernel<float, false>);
    fn<<<a.n_tokens, kThreads, 0, s>>>(d);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

}  // extern "C"
