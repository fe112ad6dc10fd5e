// Divergence of a policy from a teacher whose top logits are known, per token, and its gradient (gac_distill of
// include/gac.h).
//
// With z = logits / temperature, q = softmax(z) over the vocabulary, N the tokens that the teacher names, r the others
// taken as one, q_r = sum of q over them, p_r = 1 - sum of p:
//   top      p = softmax(teacher / temperature) over N     L = sum_N p (log p - log q)              dz = q - p
//   forward  p = exp(teacher)          L = sum_N p (log p - log q) + p_r (log p_r - log q_r)         dz = q W - p on N,
//                                      q (W - p_r / q_r) elsewhere, W = sum_N p + p_r
//   reverse  d = log q - log p         L = sum_N q d + q_r d_r                                       dz = q (d - L) on N,
//                                                                                                    q (d_r - L) elsewhere
// Every gradient outside N is exp(z) times a number of the row, so a row needs its maximum and sum outside N in one pass
// and, for the gradient, one product and one exponential per element in another.  Sums outside N are taken without the
// named tokens, which a bitmap in shared memory marks (a byte to a vector of 16 bytes): as a difference of two sums a
// small rest would be lost.  What has to do with the few named tokens, and the row's own numbers, is binary64.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cstddef>

#include "gac.h"
#include "gac_host.h"
#include "overlap.h"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kMaxSplit = 8;      // CTAs of a row: a portable cluster
constexpr float kMasked = -1e38f;      // tokens with no logit above this are taken as masked

struct DistillDev {
    const char *z;
    char *dz;
    long long z_row, dz_row;           // bytes
    const int32_t *ids;
    const char *teacher;
    long long ids_row, teacher_row;    // elements
    int teacher_bf16, kind;
    float *loss;
    const float *weights;
    uint32_t vocab, top, split;
    float c;                           // log2(e) / temperature
    double inv_temp;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float from_float(float x, float) { return x; }
__device__ __forceinline__ uint16_t from_float(float x, uint16_t) { return uint16_t(pack_bf16(x, 0.f) & 0xFFFFu); }

// 16 bytes of a row.
template <typename T>
struct Vector {
    static constexpr int N = 16 / int(sizeof(T));
    __device__ static __forceinline__ void unpack(const uint4 &x, float (&v)[N]) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : __uint_as_float(i & 1 ? w[i / 2 % 4] & 0xFFFF0000u : w[i / 2 % 4] << 16);
    }
    __device__ static __forceinline__ uint4 pack(const float (&v)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(v[i % N]) : pack_bf16(v[2 * i % N], v[(2 * i + 1) % N]);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// What a CTA knows of its part of the row.
struct Partial {
    double mass, cost;          // top: sum of e, of e (log e - z); else: sum of p, of p (log p - z) or, reverse, unused
    double named, named_cost;   // sum over named tokens of exp(z - m_named), of exp(z - m_named) (z - log p)
    float m_named, m, s;        // largest logit of named tokens; largest and sum of exp of the others'
};
// What the gradient needs of the whole row.
struct Row {
    double m, log_total, mass_scale, add, loss, weight;   // see finish()
    float m_rest, others;
};

__device__ __forceinline__ double add_lanes(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
__device__ __forceinline__ float max_lanes(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

// The row's numbers from its parts, by one thread, parts in their order.  `top_teacher`: largest value of the teacher.
__device__ void finish(const DistillDev &a, const Partial *parts, uint32_t n, double weight, Row *out) {
    double mass = 0.0, cost = 0.0, named = 0.0, named_cost = 0.0, s = 0.0;
    float m_rest = -FLT_MAX, m_named = -FLT_MAX;
    for (uint32_t i = 0; i < n; ++i) {
        m_rest = fmaxf(m_rest, parts[i].m);
        m_named = fmaxf(m_named, parts[i].m_named);
    }
    for (uint32_t i = 0; i < n; ++i) {
        mass += parts[i].mass;
        cost += parts[i].cost;
        s += double(parts[i].s) * exp((double(parts[i].m) - double(m_rest)) * a.inv_temp);
        const double f = exp((double(parts[i].m_named) - double(m_named)) * a.inv_temp);
        named += parts[i].named * f;
        named_cost += parts[i].named_cost * f;
    }
    const bool rest = m_rest > kMasked || s != s;   // a NaN is not masked
    const double m = fmax(double(m_named), rest ? double(m_rest) : -double(FLT_MAX));
    const double f_named = exp((double(m_named) - m) * a.inv_temp), f_rest = rest ? exp((double(m_rest) - m) * a.inv_temp) : 0.0;
    const double total = named * f_named + (rest ? s * f_rest : 0.0);
    const double log_total = log(total), scale = weight * a.inv_temp;
    const double lse = m * a.inv_temp + log_total;
    const double q_rest = rest ? s * f_rest / total : 0.0;
    double others = 0.0;   // q_rest times the gradient's factor outside N
    out->m = m;
    out->log_total = log_total;
    out->weight = scale;
    if (a.kind == GAC_DISTILL_TOP) {
        out->loss = cost / mass - log(mass) + lse;
        out->mass_scale = 1.0;
        out->add = 1.0 / mass;
        others = q_rest;
    } else {
        const double p_rest = fmax(1.0 - mass, 1.0 / 16777216.0);
        const double log_q_rest = rest ? (double(m_rest) - m) * a.inv_temp + log(s) - log_total : 0.0;
        if (a.kind == GAC_DISTILL_FORWARD) {
            const double w = mass + (rest ? p_rest : 0.0);
            out->loss = cost + mass * lse + (rest ? p_rest * (log(p_rest) - log_q_rest) : 0.0);
            out->mass_scale = w;
            out->add = 1.0;
            others = rest ? w * q_rest - p_rest : 0.0;
        } else {
            const double d_rest = rest ? log_q_rest - log(p_rest) : 0.0;
            out->loss = f_named / total * (named_cost - lse * named) + q_rest * d_rest;
            out->mass_scale = 0.0;
            out->add = 0.0;
            others = q_rest * (d_rest - out->loss);
        }
    }
    out->m_rest = m_rest;
    out->others = rest ? float(others / s * scale) : 0.0f;
}

template <typename T, bool GRAD>
__global__ void __launch_bounds__(kThreads)
distill_kernel(const __grid_constant__ DistillDev a) {
    using Vec = Vector<T>;
    constexpr int N = Vec::N, kFlight = 4;
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Partial parts[kMaxSplit];
    __shared__ Partial warp_part[kWarps];
    __shared__ Row row;
    __shared__ float warp_max[2][kWarps];
    __shared__ int repeated;

    const uint32_t part = a.split == 1 ? 0 : blockIdx.x % a.split, t = blockIdx.x / a.split;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, top = a.top;
    // per named token: p, or e of it; its logit, what the teacher says, which it is
    double *e_p = reinterpret_cast<double *>(dynamic);
    float *e_z = reinterpret_cast<float *>(e_p + top), *e_l = e_z + top;
    int *e_id = reinterpret_cast<int *>(e_l + top);
    uint32_t *marks = reinterpret_cast<uint32_t *>(e_id + top);

    const char *z = a.z + (long long)t * a.z_row;
    char *dz = GRAD ? a.dz + (long long)t * a.dz_row : nullptr;
    // the row in vectors of 16 bytes: element v is at place v + off
    const uint32_t off = uint32_t(reinterpret_cast<uint64_t>(z) / sizeof(T)) % N;
    const uint32_t vectors = (a.vocab + off + N - 1) / N, per = (vectors + a.split - 1) / a.split;
    const uint32_t lo = min(part * per, vectors), hi = min(lo + per, vectors);
    const uint32_t first = max(lo * N, off) - off, last = max(min(hi * N, a.vocab + off), off) - off;   // elements of this part
    // vectors that are whole: the row's first and last may not be
    const uint32_t whole_lo = max(lo, off ? 1u : 0u), whole_hi = min(hi, (a.vocab + off) / N);
    auto mark_of = [&](uint32_t vector) { return reinterpret_cast<const uint8_t *>(marks)[vector - lo]; };

    for (uint32_t i = threadIdx.x; i < (hi - lo + 3) / 4; i += kThreads) marks[i] = 0;
    if (threadIdx.x == 0) repeated = 0;
    __syncthreads();

    // ---- what the teacher names
    bool any = false;
    float most = -INFINITY, m_named = -FLT_MAX;
    for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
        int id = a.ids[(long long)t * a.ids_row + i];
        const long long at = (long long)t * a.teacher_row + i;
        const float l = a.teacher_bf16 ? as_float(reinterpret_cast<const uint16_t *>(a.teacher)[at]) : reinterpret_cast<const float *>(a.teacher)[at];
        if (id < 0 || uint32_t(id) >= a.vocab || l == -INFINITY) id = -1;
        e_id[i] = id;
        e_l[i] = l;
        if (id < 0) continue;
        any = true;
        most = l > most || l != l ? l : most;
        if (uint32_t(id) >= first && uint32_t(id) < last) {
            const float x = as_float(reinterpret_cast<const T *>(z)[id]);
            e_z[i] = x;
            m_named = fmaxf(m_named, x);
            const uint32_t place = uint32_t(id) + off - lo * N;   // from the start of this part
            const uint32_t bit = 1u << (place / N % 4 * 8 + place % N);
            if (atomicOr(marks + place / N / 4, bit) & bit) repeated = 1;
        }
    }
    any = __syncthreads_or(any);
    const float weight = a.weights ? a.weights[t] : 1.0f;
    if (!any) {   // nothing to compare with: the row is not read
        if (a.loss && part == 0 && threadIdx.x == 0) a.loss[t] = 0.0f;
        if (GRAD)
            for (uint32_t v = first + threadIdx.x; v < last; v += kThreads) reinterpret_cast<T *>(dz)[v] = T(0);
        return;
    }
    if (a.split > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");   // this CTA has started
    if (repeated) {   // of several with the same token the first counts
        for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
            const int id = e_id[i];
            bool again = false;
            for (uint32_t j = 0; id >= 0 && j < i; ++j) again |= e_id[j] == id;
            e_p[i] = again ? 1.0 : 0.0;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < top; i += kThreads)
            if (e_p[i] != 0.0) e_id[i] = -1;
    }
    most = max_lanes(most);
    m_named = max_lanes(m_named);
    if (lane == 0) {
        warp_max[0][warp] = most;
        warp_max[1][warp] = m_named;
    }
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) {
        most = fmaxf(most, warp_max[0][i]);
        m_named = fmaxf(m_named, warp_max[1][i]);
    }
    Partial mine = {};
    for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
        const int id = e_id[i];
        if (id < 0 || uint32_t(id) < first || uint32_t(id) >= last) continue;
        const double x = double(e_z[i]) * a.inv_temp;
        const double l = a.kind == GAC_DISTILL_TOP ? (double(e_l[i]) - double(most)) * a.inv_temp : double(e_l[i]);
        const double p = exp(l), q = exp((double(e_z[i]) - double(m_named)) * a.inv_temp);
        e_p[i] = p;
        mine.mass += p;
        mine.cost += p > 0.0 ? p * (l - x) : p;     // 0 log 0 = 0; a NaN stays one
        mine.named += q;
        mine.named_cost += q > 0.0 ? q * (x - l) : q;
    }

    // ---- largest logit and sum of exponentials of all others
    float m = -FLT_MAX, s = 0.0f;
    auto take = [&](float (&v)[N], uint32_t marked) {
        if (marked) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (marked >> i & 1u) v[i] = -INFINITY;
        }
    };
    auto add = [&](const float (&v)[N]) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) sum += exp2_fast((v[i] - m) * a.c);
        s += sum;
    };
    auto raise = [&](float top_of) {
        const float next = fmaxf(m, top_of);
        s *= exp2_fast((m - next) * a.c);
        m = next;
    };
    const uint4 *zv = reinterpret_cast<const uint4 *>(z - (long long)off * (long long)sizeof(T));
    for (uint32_t j = whole_lo + threadIdx.x; j < whole_hi; j += kFlight * kThreads) {
        uint4 x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (j + u * kThreads < whole_hi) x[u] = __ldcg(zv + j + u * kThreads);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            if (j + u * kThreads >= whole_hi) break;
            float v[N], best = -FLT_MAX;
            Vec::unpack(x[u], v);
            take(v, mark_of(j + u * kThreads));
#pragma unroll
            for (int i = 0; i < N; ++i) best = fmaxf(best, v[i]);
            raise(best);
            add(v);
        }
    }
    // a vector of the row that is not whole: its elements, by one thread each
    auto edge = [&](auto each) {
        const uint32_t head = min(whole_lo * N > off ? whole_lo * N - off : 0u, last), tail = max(whole_hi * N > off ? whole_hi * N - off : 0u, head);
        if (first + threadIdx.x < head) each(first + threadIdx.x);
        if (tail + threadIdx.x < last) each(tail + threadIdx.x);
    };
    auto marked_element = [&](uint32_t v) { return mark_of((v + off) / N) >> ((v + off) % N) & 1u; };
    edge([&](uint32_t v) {
        if (marked_element(v)) return;
        const float x = as_float(reinterpret_cast<const T *>(z)[v]);
        raise(x);
        s += exp2_fast((x - m) * a.c);
    });
    const float m_all = max_lanes(m);
    s *= exp2_fast((m - m_all) * a.c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    mine.mass = add_lanes(mine.mass);
    mine.cost = add_lanes(mine.cost);
    mine.named = add_lanes(mine.named);
    mine.named_cost = add_lanes(mine.named_cost);
    mine.m = m_all;
    mine.s = s;
    if (lane == 0) warp_part[warp] = mine;
    __syncthreads();
    if (a.split > 1) asm volatile("barrier.cluster.wait;" ::: "memory");             // all have: their memory may be written
    if (threadIdx.x == 0) {
        Partial sum = warp_part[0];
        for (int i = 1; i < kWarps; ++i) sum.m = fmaxf(sum.m, warp_part[i].m);
        sum.s = 0.0f;
        for (int i = 0; i < kWarps; ++i) sum.s += warp_part[i].s * exp2_fast((warp_part[i].m - sum.m) * a.c);
        for (int i = 1; i < kWarps; ++i) {
            sum.mass += warp_part[i].mass;
            sum.cost += warp_part[i].cost;
            sum.named += warp_part[i].named;
            sum.named_cost += warp_part[i].named_cost;
        }
        sum.m_named = m_named;
        if (a.split == 1) {
            parts[0] = sum;
        } else {   // to all parts of the row
            cg::cluster_group cluster = cg::this_cluster();
            for (uint32_t i = 0; i < a.split; ++i) *cluster.map_shared_rank(&parts[part], i) = sum;
        }
    }
    if (a.split > 1) cg::this_cluster().sync();
    if (threadIdx.x == 0) {
        Row r;
        finish(a, parts, a.split, double(weight), &r);
        if (a.loss && part == 0) a.loss[t] = float(r.loss);
        row = r;
    }
    if (!GRAD) return;
    __syncthreads();

    // ---- gradient
    const float m_rest = row.m_rest, others = row.others;
    auto grad = [&](float x) { return exp2_fast((x - m_rest) * a.c) * others; };
    const bool aligned = (reinterpret_cast<uint64_t>(dz) - reinterpret_cast<uint64_t>(z)) % 16 == 0;
    for (uint32_t j = whole_lo + threadIdx.x; j < whole_hi; j += kFlight * kThreads) {
        uint4 x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (j + u * kThreads < whole_hi) x[u] = __ldcs(zv + j + u * kThreads);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            if (j + u * kThreads >= whole_hi) break;
            float v[N];
            Vec::unpack(x[u], v);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = grad(v[i]);
            const uint32_t at = (j + u * kThreads) * N - off;
            if (aligned) {
                *reinterpret_cast<uint4 *>(dz + (long long)at * (long long)sizeof(T)) = Vec::pack(v);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) reinterpret_cast<T *>(dz)[at + i] = from_float(v[i], T{});
            }
        }
    }
    edge([&](uint32_t v) { reinterpret_cast<T *>(dz)[v] = from_float(grad(as_float(reinterpret_cast<const T *>(z)[v])), T{}); });
    __syncthreads();   // the named tokens' own gradients over what has been written
    for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
        const int id = e_id[i];
        if (id < 0 || uint32_t(id) < first || uint32_t(id) >= last) continue;
        const double log_q = (double(e_z[i]) - row.m) * a.inv_temp - row.log_total, q = exp(log_q);
        double g;
        if (a.kind == GAC_DISTILL_REVERSE) {
            g = q == 0.0 ? 0.0 : q * (log_q - double(e_l[i]) - row.loss);
        } else {
            g = q * row.mass_scale - e_p[i] * row.add;
        }
        reinterpret_cast<T *>(dz)[id] = from_float(float(g * row.weight), T{});
    }
}

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

}  // namespace

extern "C" {

int gac_distill(const gac_distill_args *args, int cuda_device, void *cuda_stream) {
    if (!args) return fail(nullptr, GAC_ERR_INVALID_ARG, "args is NULL%s");
    const gac_distill_args &a = *args;
    if (a.dtype != GAC_F32 && a.dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "logits are float32 or bfloat16%s");
    if (a.teacher_dtype != GAC_F32 && a.teacher_dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "the teacher's values are float32 or bfloat16%s");
    if (a.kind < GAC_DISTILL_TOP || a.kind > GAC_DISTILL_REVERSE) return fail(nullptr, GAC_ERR_INVALID_ARG, "unknown kind%s");
    if (a.reserved != 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "reserved must be 0%s");
    if (!(a.temperature > 0.0) || !isfinite(a.temperature) || !(a.temperature >= 1e-3 && a.temperature <= 1e3))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "temperature must be 1e-3..1e3%s");
    if (a.vocab < 1 || a.vocab > GAC_DISTILL_MAX_VOCAB) return fail(nullptr, GAC_ERR_INVALID_ARG, "vocab must be 1..%s%lld", "", (long long)GAC_DISTILL_MAX_VOCAB);
    if (a.top < 1 || a.top > GAC_DISTILL_MAX_TOP) return fail(nullptr, GAC_ERR_INVALID_ARG, "top must be 1..%s%lld", "", GAC_DISTILL_MAX_TOP);
    if (a.n_tokens > (1u << 27)) return fail(nullptr, GAC_ERR_INVALID_ARG, "n_tokens out of range%s");
    if (a.n_tokens == 0) return GAC_OK;
    if (!a.loss && !a.d_logits) return fail(nullptr, GAC_ERR_INVALID_ARG, "neither loss nor d_logits is wanted%s");
    const uint64_t size = a.dtype == GAC_BF16 ? 2 : 4, t_size = a.teacher_dtype == GAC_BF16 ? 2 : 4;
    auto off = [](const void *p, uint64_t n) { return reinterpret_cast<uint64_t>(p) % n != 0; };
    if (!a.logits || !a.ids || !a.teacher || off(a.logits, size) || off(a.d_logits, size) || off(a.ids, 4) || off(a.teacher, t_size) ||
        off(a.loss, 4) || off(a.weights, 4))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "a pointer is NULL or misaligned%s");
    const int64_t most = int64_t(1) << 40;
    auto bad = [&](int64_t stride) { return stride < 0 || stride > most; };
    if (bad(a.logits_row) || bad(a.d_row) || bad(a.ids_row) || bad(a.teacher_row))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "strides must be 0..2^40 elements%s");
    auto rows = [&](const void *p, int64_t stride, uint64_t n, uint64_t bytes) {
        return Rows{reinterpret_cast<uint64_t>(p), uint64_t(stride) * bytes, 0, a.n_tokens, 1, n * bytes};
    };
    const Rows in[4] = {rows(a.logits, a.logits_row, a.vocab, size), rows(a.ids, a.ids_row, a.top, 4),
                        rows(a.teacher, a.teacher_row, a.top, t_size), rows(a.weights, 1, 1, 4)};
    Rows out[2];
    int outs = 0;
    if (a.loss) out[outs++] = rows(a.loss, 1, 1, 4);
    if (a.d_logits) {
        if (a.n_tokens > 1 && a.d_row < int64_t(a.vocab)) return fail(nullptr, GAC_ERR_INVALID_ARG, "rows of the gradient overlap one another%s");
        out[outs++] = rows(a.d_logits, a.d_row, a.vocab, size);
        if (a.loss && share(out[0], out[1])) return fail(nullptr, GAC_ERR_INVALID_ARG, "loss and gradient overlap%s");
    }
    for (int i = 0; i < outs; ++i)
        for (int j = 0; j < (a.weights ? 4 : 3); ++j) {
            const bool in_place = j == 0 && out[i].p == in[0].p && a.d_logits == a.logits && a.d_row == a.logits_row;
            if (!in_place && share(out[i], in[j])) return fail(nullptr, GAC_ERR_INVALID_ARG, "an output overlaps an input without being in place%s");
        }
    DistillDev d;
    d.z = static_cast<const char *>(a.logits);
    d.dz = static_cast<char *>(a.d_logits);
    d.z_row = a.logits_row * int64_t(size);
    d.dz_row = a.d_row * int64_t(size);
    d.ids = a.ids;
    d.teacher = static_cast<const char *>(a.teacher);
    d.ids_row = a.ids_row;
    d.teacher_row = a.teacher_row;
    d.teacher_bf16 = a.teacher_dtype == GAC_BF16;
    d.kind = a.kind;
    d.loss = a.loss;
    d.weights = a.weights;
    d.vocab = a.vocab;
    d.top = a.top;
    d.inv_temp = 1.0 / a.temperature;
    d.c = float(M_LOG2E / a.temperature);
    // Few rows are split over a cluster, as long as a part has some thousands of elements.
    d.split = 1;
    while (d.split < kMaxSplit && uint64_t(a.n_tokens) * d.split < 148 * 4 && a.vocab / (2 * d.split) >= 4096) d.split *= 2;
    const uint32_t vec = 16 / uint32_t(size), vectors = (a.vocab + 2 * vec - 2) / vec, per = (vectors + d.split - 1) / d.split;
    const size_t smem = size_t(a.top) * 20 + (per + 3) / 4 * 4;
    Range range("gac_distill");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    void (*fn)(const DistillDev) = nullptr;
    if (a.dtype == GAC_BF16) fn = a.d_logits ? distill_kernel<uint16_t, true> : distill_kernel<uint16_t, false>;
    else fn = a.d_logits ? distill_kernel<float, true> : distill_kernel<float, false>;
    if (smem > 40 * 1024) GAC_CUDA(nullptr, cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)));
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3(a.n_tokens * d.split);
    how.blockDim = dim3(kThreads);
    how.dynamicSmemBytes = smem;
    how.stream = static_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = d.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    how.attrs = attr;
    how.numAttrs = 1;
    GAC_CUDA(nullptr, cudaLaunchKernelEx(&how, fn, d));
    return GAC_OK;
}

}  // extern "C"
