// What the operators on query and key heads share (rotary.cu, norm_rotary.cu): where a token stands, its sines and
// cosines, vectors of elements, and the checks of their arguments.
#pragma once

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
static_assert(GAC_ROTARY_MAX_AXES == 4, "an axis is kept in two bits");

struct RotaryDev {
    const char *x[2];
    char *y[2];
    long long x_token[2], x_head[2], y_token[2], y_head[2];
    uint32_t heads[2];
    uint32_t n_tokens, n_seqs, head_dim, pairs;
    const int32_t *positions, *cu;
    long long axis_stride;                          // 0: one axis turns all pairs
    uint32_t axis[GAC_ROTARY_MAX_DIM / 2 / 16];     // the axis of each pair, two bits
    float scale;
    int inverse;
    double turns[GAC_ROTARY_MAX_DIM / 2];           // turns per position of each pair
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

// Cosine and sine, already scaled, of a pair at a position.
__device__ __forceinline__ float2 turn_of(const RotaryDev &a, uint32_t pair, int pos) {
    const double turns = double(pos) * a.turns[pair];
    float s, c;
    sincospif(2.0f * float(turns - rint(turns)), &s, &c);
    return make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
}
__device__ __forceinline__ int position_on_axis(const RotaryDev &a, uint32_t pair, uint32_t t) {
    return a.positions[(a.axis[pair / 16] >> (2 * (pair % 16)) & 3u) * a.axis_stride + t];
}
// Of every pair of the CTA's token.  AXES: its pairs may be turned by different axes.
template <bool AXES>
__device__ __forceinline__ void fill_wheel(const RotaryDev &a, float2 *wheel, uint32_t t) {
    for (uint32_t i = threadIdx.x; i < a.pairs; i += kThreads) {
        const int pos = !a.positions ? place_in_sequence(a.cu, a.n_seqs, t) : AXES ? position_on_axis(a, i, t) : a.positions[t];
        wheel[i] = turn_of(a, i, pos);
    }
    __syncthreads();
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

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

Rows rows_of(const void *p, int64_t token, int64_t head, uint64_t nt, uint64_t nh, uint64_t dim, uint64_t size) {
    return Rows{reinterpret_cast<uint64_t>(p), uint64_t(token) * size, uint64_t(head) * size, nt, nh, dim * size};
}

// Checks the arguments and fills `d`; x and y are the heads as blocks of rows, for those that are there.  GAC_OK with
// nothing to do leaves n_tokens or both head counts at 0.  `norm`: nothing need be turned, and never the other way.
int check_rotary(const gac_rotary_args &a, const gac_rotary_axes *axes, bool norm, RotaryDev &d, Rows (&x)[2], Rows (&y)[2]) {
    if (a.dtype != GAC_F32 && a.dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "heads are float32 or bfloat16%s");
    if (a.layout != GAC_ROTARY_HALF && a.layout != GAC_ROTARY_INTERLEAVED) return fail(nullptr, GAC_ERR_INVALID_ARG, "unknown layout%s");
    if ((a.inverse != 0 && a.inverse != 1) || a.reserved != 0)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "inverse must be 0 or 1, reserved 0%s");
    if ((a.rot_dim < 2 && !(norm && a.rot_dim == 0)) || a.rot_dim % 2 || a.rot_dim > a.head_dim || a.rot_dim > GAC_ROTARY_MAX_DIM)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "rot_dim must be even, at least 2 (norms: or 0), at most head_dim and %s%lld", "", GAC_ROTARY_MAX_DIM);
    if (a.head_dim > 1024 || a.heads[0] > 4096 || a.heads[1] > 4096 || a.n_tokens > (1u << 30) || a.n_seqs > (1u << 30))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "head_dim, heads or n_tokens out of range%s");
    if (!a.freqs && a.rot_dim) return fail(nullptr, GAC_ERR_INVALID_ARG, "freqs is NULL%s");
    if (!isfinite(a.scale)) return fail(nullptr, GAC_ERR_INVALID_ARG, "scale must be finite%s");
    const uint64_t size = a.dtype == GAC_BF16 ? 2 : 4;
    int both = 0;
    d.axis_stride = 0;
    memset(d.axis, 0, sizeof(d.axis));
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
    if (axes) {
        if (axes->n_axes < 1 || axes->n_axes > GAC_ROTARY_MAX_AXES || axes->reserved != 0)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "n_axes must be 1..%s%lld, reserved 0", "", GAC_ROTARY_MAX_AXES);
        if (axes->stride < 0 || axes->stride > int64_t(1) << 40)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "the stride of the axes' positions must be 0..2^40 elements%s");
        if (!axes->axis) return fail(nullptr, GAC_ERR_INVALID_ARG, "axis is NULL%s");
        d.axis_stride = axes->stride;
        for (uint32_t i = 0; i < a.rot_dim / 2; ++i) {
            if (axes->axis[i] >= axes->n_axes) return fail(nullptr, GAC_ERR_INVALID_ARG, "the axis of pair %s%lld is out of range", "", i);
            d.axis[i / 16] |= uint32_t(axes->axis[i]) << (2 * (i % 16));
        }
    }
    if (a.n_tokens == 0 || (a.heads[0] == 0 && a.heads[1] == 0)) return GAC_OK;
    if (axes && !a.positions) return fail(nullptr, GAC_ERR_INVALID_ARG, "axes need positions%s");
    if (a.rot_dim && !a.positions && (!a.cu_seqlens || reinterpret_cast<uint64_t>(a.cu_seqlens) % 4))
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
    return GAC_OK;
}

// Whether every vector of n elements of every head starts on a boundary of its size and ends inside its part of the head.
bool vectors_fit(const RotaryDev &d, uint32_t n, uint64_t size) {
    const uint64_t bytes = n * size;
    if (d.pairs % n || d.head_dim % n) return false;
    for (int w = 0; w < 2; ++w)
        if (d.heads[w] && (reinterpret_cast<uint64_t>(d.x[w]) % bytes || reinterpret_cast<uint64_t>(d.y[w]) % bytes || d.x_token[w] % n ||
                           d.x_head[w] % n || d.y_token[w] % n || d.y_head[w] % n))
            return false;
    return true;
}

}  // namespace
