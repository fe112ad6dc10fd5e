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
// named tokens, which are overwritten with -infinity before: as a difference of two sums a small rest would be lost.
// What has to do with the few named tokens, and the row's own numbers, is binary64.
//
// One CTA to a row, or, where rows are few or long, a cluster of up to eight that exchange what they know of their parts
// through distributed shared memory.  The second pass reads the row again, backwards and out of L2: rows are loaded with
// evict-last, read again and written with evict-first, and cut into so many parts that the rows in use fit.  Loads go through a
// ring in shared memory, because what bounds the kernel is bytes in flight beside the chain from a row's last load to its first
// gradient (sums over the CTA, exponentials and logarithms in binary64, about 5 us), which the SM's other CTAs have to cover.
// Measured, ten calls after a pause: 4096 x 151936 bfloat16 with the gradient 434 us (5.7 TB/s of one read and one write, 0.89 of a
// plain copy's rate; memory reads the logits 1.14 times), 8191 x 32000 float32, a quarter without a teacher, 310 (0.92), 2048 x 151936
// values alone 105 (0.92).  In a second of calls on end, under the power cap, 503, 330 and 119.  A row held in the shared memory of eight
// CTAs took 618 where this took 444, and persistent CTAs that read the next row while parts of the last are exchanged 1490.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cstddef>

#include "gac.h"
#include "gac_host.h"
#include "overlap.h"
#include "sm100.cuh"

namespace {

namespace cg = cooperative_groups;

// Threads of a CTA, CTAs of an SM that registers are left for, and the ring: groups of vectors that a thread loads at once.  Short rows
// take smaller CTAs: what a row takes beside its loads is the same for all, and more rows at once cover it (4096 rows of 64 kB with the
// gradient 100 us, with the other shape 111; values alone 52 and 76; 4096 rows of 304 kB with the gradient 472 and 434, values alone the
// same).  Of long rows with the gradient four CTAs fit an SM while a CTA's part of a row has about 90 kB, with the marks of more three.
template <bool GRAD, bool SHORT>
struct Shape {
    static constexpr int kThreads = SHORT ? 128 : GRAD ? 256 : 384, kCtas = SHORT ? 8 : GRAD ? 4 : 3, kWarps = kThreads / 32;
    static constexpr int kFlight = !SHORT && GRAD ? 3 : 4, kRing = !SHORT && GRAD ? 4 : 2, kRingBytes = kRing * kFlight * kThreads * 16;
};
constexpr uint32_t kMaxSplit = 8;      // CTAs of a row: a portable cluster
constexpr uint64_t kInUse = 96u << 20; // bytes of rows in use at once, of 126 MB of L2
// The ring, the most named tokens, and marks: a byte to 16 bytes of a row, or, where it is split, of an eighth of it.
constexpr size_t kMaxSmem = Shape<false, false>::kRingBytes + GAC_DISTILL_MAX_TOP * 28 + GAC_DISTILL_MAX_ROW_BYTES / 16 + 16;
static_assert(kMaxSmem <= 224 * 1024 && Shape<true, false>::kRingBytes <= Shape<false, false>::kRingBytes, "fits an SM");
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
    uint32_t vocab, top, split, mark_words;
    float c;                           // log2(e) / temperature, rounded;
    double c_off;                      // what it lacks, times log(2)
    double inv_temp;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }
__device__ __forceinline__ float from_float(float x, float) { return x; }
__device__ __forceinline__ uint16_t from_float(float x, uint16_t) { return uint16_t(bf16x2(x, 0.f) & 0xFFFFu); }

// 16 bytes of a row.
template <typename T>
struct Vector {
    static constexpr int N = 16 / int(sizeof(T));
    static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;   // -infinity throughout
    __device__ static __forceinline__ void unpack(const uint4 &x, float2 (&v)[N / 2]) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            v[i] = sizeof(T) == 4 ? make_float2(__uint_as_float(w[2 * i % 4]), __uint_as_float(w[(2 * i + 1) % 4]))
                                  : make_float2(__uint_as_float(w[i % 4] << 16), __uint_as_float(w[i % 4] & 0xFFFF0000u));
    }
    __device__ static __forceinline__ uint4 pack(const float2 (&v)[N / 2]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = sizeof(T) == 4 ? __float_as_uint(i & 1 ? v[i / 2].y : v[i / 2].x) : bf16x2(v[i % (N / 2)].x, v[i % (N / 2)].y);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the larger of two vectors, element by element, NaN where both are; and the largest element, -FLT_MAX at least
    __device__ static __forceinline__ uint4 larger(const uint4 &a, const uint4 &b) {
        return make_uint4(two(a.x, b.x), two(a.y, b.y), two(a.z, b.z), two(a.w, b.w));
    }
    __device__ static __forceinline__ float largest(const uint4 &a) {
        const uint32_t w = two(two(a.x, a.y), two(a.z, a.w));
        if (sizeof(T) == 4) return fmaxf(__uint_as_float(w), -FLT_MAX);
        return fmaxf(fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)), -FLT_MAX);
    }
    // -infinity in the place of the marked elements
    __device__ static __forceinline__ uint4 without(const uint4 &x, uint32_t marked) {
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (marked >> i & 1u) {
                if (sizeof(T) == 4) w[i % 4] = kNone;
                else w[i / 2 % 4] = i & 1 ? (w[i / 2 % 4] & 0xFFFFu) | 0xFF800000u : (w[i / 2 % 4] & 0xFFFF0000u) | 0xFF80u;
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __forceinline__ uint32_t two(uint32_t a, uint32_t b) {
        uint32_t r;
        if (sizeof(T) == 4) asm("max.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
};

// Sums of exponentials are kept as multiples of 2^level, level a whole number next to the product of the largest logit and c, so that
// they are brought together exactly.  Up to kFar a rounded product is off by at most 64, so that no power leaves binary32.  Levels
// stop there: what is masked far below adds nothing to a sum that ordinary logits are in, and a row whose own largest is beyond is a far row.
constexpr float kFar = 2147483648.0f;
__device__ __forceinline__ float level_of(float m, float c) { return rintf(fminf(fmaxf(m * c, -kFar), kFar)); }
__device__ __forceinline__ bool is_far(float m, float c) { return fabsf(m * c) > kFar; }
__device__ __forceinline__ double power_of_two(float whole) {   // 0 or less
    return whole < -1000.0f ? 0.0 : __hiloint2double((1023 + int(whole)) << 20, 0);
}
// What a CTA, or a warp, knows of its part of the row.
struct Partial {
    double mass, cost;          // top: sum of e, of e (log e - z); else: sum of p, of p (log p - z)
    double named, named_cost;   // sum over named tokens of exp(z), of exp(z) (z - log p), in units of 2^level_of(named_m)
    float named_m;              // their largest logit
    float m, s;                 // of the others the largest logit, and the sum of exp(z) in units of 2^level_of(m)
};
// What the gradient needs of the whole row.
struct Row {
    double lse, total;          // log q = z - lse; the sum of exp(z) in units of 2^unit
    double q_scale, p_scale;    // of a named token's q and p (top, forward)
    double loss, weight;
    float unit;
    float level, others;        // elsewhere: 2^(logit c - level) others
    float m, named_m;           // the largest logits, elsewhere and of named tokens
    int far;
};

template <typename F>
__device__ __forceinline__ F add_lanes(F x, int from) {
#pragma unroll
    for (int o = from; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
__device__ __forceinline__ float max_lanes(float x, int from) {
#pragma unroll
    for (int o = from; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}
// No part at all.
__device__ __forceinline__ Partial no_part() {
    Partial p = {};
    p.m = p.named_m = -FLT_MAX;
    return p;
}
// The sum of `n` parts, a power of two, one to a lane of every n, in all lanes.
__device__ __forceinline__ Partial add_parts(Partial p, const DistillDev &a, int n) {
    const float m = max_lanes(p.m, n / 2), named_m = max_lanes(p.named_m, n / 2);
    p.s = add_lanes(p.s * exp2_approx(level_of(p.m, a.c) - level_of(m, a.c)), n / 2);
    const double f = power_of_two(level_of(p.named_m, a.c) - level_of(named_m, a.c));
    p.mass = add_lanes(p.mass, n / 2);
    p.cost = add_lanes(p.cost, n / 2);
    p.named = add_lanes(p.named * f, n / 2);
    p.named_cost = add_lanes(p.named_cost * f, n / 2);
    p.m = m;
    p.named_m = named_m;
    return p;
}

// The row's numbers from the sum of its parts, by a whole warp: what the gradient outside N needs first (`rest` and `s` for the rest).
struct Sums {
    double s, f_rest, f_named, p_rest;
    double unit, rest_unit;     // logarithms: of what total is a multiple of, and of what s is, relative to it
    bool rest;
};
__device__ __forceinline__ double what_is_left(double mass) { return 1.0 - mass < 1.0 / 16777216.0 ? 1.0 / 16777216.0 : 1.0 - mass; }   // NaN of NaN
__device__ __forceinline__ bool has_rest(const Partial &p) { return p.m > kMasked || p.s != p.s; }   // a NaN is not masked
// Whether the largest logit of what counts is beyond the levels: m outside N, named_m in it.
__device__ __forceinline__ bool far_row(const DistillDev &a, float m, float named_m) {
    return (m > kMasked ? is_far(m, a.c) : is_far(named_m, a.c)) || named_m * a.c > kFar;
}
__device__ __forceinline__ Sums start(const DistillDev &a, const Partial &p, Row &r) {
    Sums x;
    x.rest = has_rest(p);
    const float named_level = level_of(p.named_m, a.c);
    r.level = level_of(p.m, a.c);
    r.unit = x.rest ? fmaxf(named_level, r.level) : named_level;
    x.unit = double(r.unit) * M_LN2;
    x.rest_unit = double(r.level - r.unit) * M_LN2;
    x.f_rest = x.rest ? power_of_two(r.level - r.unit) : 0.0;
    x.f_named = power_of_two(named_level - r.unit);
    // powers were taken of logit c, and c is rounded: near the largest logit they are off by this
    const double off = double(p.m) * a.c_off;
    x.s = !x.rest ? 0.0 : double(p.s) * (fabs(off) < 0.01 ? 1.0 + off * (1.0 + off * (0.5 + off * (1.0 / 6.0))) : exp(off));
    const double total = p.named * x.f_named + x.s * x.f_rest;
    r.total = total < double(INFINITY) ? total : double(NAN);
    x.p_rest = what_is_left(p.mass);
    return x;
}
__device__ __forceinline__ float factor(double others, const Sums &x, const Partial &p, const Row &r) {
    return x.rest ? float(others) / p.s * float(r.weight) : 0.0f;
}
__device__ __forceinline__ void finish_gradient(const DistillDev &a, const Partial &p, const Sums &x, Row &r) {   // top, forward
    const double q_rest = x.s * x.f_rest / r.total;
    const bool top = a.kind == GAC_DISTILL_TOP;
    r.q_scale = top ? 1.0 : p.mass + (x.rest ? x.p_rest : 0.0);
    r.p_scale = top ? 1.0 / p.mass : 1.0;
    r.others = factor(top ? q_rest : r.q_scale * q_rest - x.p_rest, x, p, r);
}
__device__ __forceinline__ void finish_loss(const DistillDev &a, const Partial &p, const Sums &x, Row &r) {
    const uint32_t all = 0xFFFFFFFFu, which = threadIdx.x & 3;
    const double l = log(which == 0 ? r.total : which == 1 ? x.s : which == 2 ? x.p_rest : p.mass);
    const double log_total = __shfl_sync(all, l, 0), log_s = __shfl_sync(all, l, 1), log_p_rest = __shfl_sync(all, l, 2), log_mass = __shfl_sync(all, l, 3);
    r.lse = x.unit + log_total;
    const double log_q_rest = x.rest ? x.rest_unit + log_s - log_total : 0.0;
    if (a.kind == GAC_DISTILL_TOP) {
        r.loss = p.cost / p.mass - log_mass + r.lse;
    } else if (a.kind == GAC_DISTILL_FORWARD) {
        r.loss = p.cost + p.mass * r.lse + (x.rest ? x.p_rest * (log_p_rest - log_q_rest) : 0.0);
    } else {
        const double q_rest = x.s * x.f_rest / r.total, d_rest = x.rest ? log_q_rest - log_p_rest : 0.0;
        r.loss = x.f_named / r.total * (p.named_cost - r.lse * p.named) + q_rest * d_rest + 0.0 * p.mass;   // a NaN that nothing weighs stays one
        r.others = factor(q_rest * (d_rest - r.loss), x, p, r);
    }
}

// One CTA's part of a row.
struct Span {
    const char *z;              // place 0; element v of the row is at place v + off, 16 bytes make a vector
    uint32_t off, end;          // places off .. end - 1 are the row's
    uint32_t vectors, lo, hi;   // the row's vectors; this part's
    uint32_t whole_lo, whole_hi;   // those of this part that are whole: the row's first and last may not be
};
template <typename T>
__device__ __forceinline__ Span span_of(const DistillDev &a, uint32_t t, uint32_t part) {
    constexpr uint32_t N = Vector<T>::N;
    Span s;
    const char *z = a.z + (long long)t * a.z_row;
    s.off = uint32_t(reinterpret_cast<uint64_t>(z) / sizeof(T)) % N;
    s.z = z - s.off * sizeof(T);
    s.end = a.vocab + s.off;
    s.vectors = (s.end + N - 1) / N;
    const uint32_t per = (s.vectors + a.split - 1) / a.split;
    s.lo = min(part * per, s.vectors);
    s.hi = min(s.lo + per, s.vectors);
    s.whole_lo = max(s.lo, s.off ? 1u : 0u);
    s.whole_hi = min(s.hi, s.end / N);
    return s;
}

// The named tokens of a CTA's part, in its dynamic shared memory: p, or e of it; exp(z); the logit, what the teacher says, the place in
// the row (kNowhere: not of this part, or absent); then a byte to a vector, a bit to an element: which are named.
constexpr uint32_t kNowhere = 0xFFFFFFFFu;
struct Named {
    double *p, *q;
    float *z, *l;
    uint32_t *at, *marks;
    __device__ __forceinline__ Named(char *from, uint32_t top) {
        p = reinterpret_cast<double *>(from);
        q = p + top;
        z = reinterpret_cast<float *>(q + top);
        l = z + top;
        at = reinterpret_cast<uint32_t *>(l + top);
        marks = at + top;
    }
};
// A warp's share of them, with z = (logit - base) / temperature and exp(z) in units of exp(unit); `most`: the largest that the teacher says.
__device__ __forceinline__ Partial add_named(const DistillDev &a, const Named &e, uint32_t threads, float most, double base, double unit) {
    Partial mine = {};
    for (uint32_t i = threadIdx.x; i < a.top; i += threads) {
        if (e.at[i] == kNowhere) continue;
        const double z = (double(e.z[i]) - base) * a.inv_temp, says = e.l[i];
        const double log_p = a.kind == GAC_DISTILL_TOP ? (says - double(most)) * a.inv_temp : says;
        const double p = exp(log_p), q = exp(z - unit);
        e.p[i] = p;
        e.q[i] = q;
        mine.mass += p;
        mine.cost += p > 0.0 ? p * (log_p - z) : p;     // 0 log 0 = 0; a NaN stays one
        mine.named += q;
        mine.named_cost += q > 0.0 ? q * (z - log_p) : q;
    }
    if (__any_sync(0xFFFFFFFFu, mine.named != 0.0 || mine.mass != 0.0)) {
        mine.mass = add_lanes(mine.mass, 16);
        mine.cost = add_lanes(mine.cost, 16);
        mine.named = add_lanes(mine.named, 16);
        mine.named_cost = add_lanes(mine.named_cost, 16);
    }
    return mine;
}
// The parts of a row brought together by every CTA's warp 0; all have arrived at the cluster's barrier before, and their `parts` may be written.
__device__ __forceinline__ Partial exchange(Partial sum, const DistillDev &a, Partial *parts, uint32_t part) {
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (warp == 0) {
        if (lane < a.split) *cg::this_cluster().map_shared_rank(&parts[part], lane) = sum;
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    } else {
        asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    }
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    return warp == 0 ? add_parts(lane % kMaxSplit < a.split ? parts[lane % kMaxSplit] : no_part(), a, kMaxSplit) : sum;
}
// The named tokens' gradients, over what has been written in their places.
template <typename T>
__device__ __forceinline__ void put_named(const DistillDev &a, const Named &e, const Row &row, uint32_t threads, char *dz, double base, double f) {
    for (uint32_t i = threadIdx.x; i < a.top; i += threads) {
        if (e.at[i] == kNowhere) continue;
        const double q = e.q[i] * f / row.total;
        double g = q * row.q_scale - e.p[i] * row.p_scale;
        if (a.kind == GAC_DISTILL_REVERSE) g = q == 0.0 ? 0.0 : q * ((double(e.z[i]) - base) * a.inv_temp - row.lse - double(e.l[i]) - row.loss);
        reinterpret_cast<T *>(dz)[e.at[i]] = from_float(float(g * row.weight), T{});
    }
}

// What the teacher says of an entry, and whether it is there.
__device__ __forceinline__ void read_entry(const DistillDev &a, uint32_t t, uint32_t i, int &id, float &says) {
    id = a.ids[(long long)t * a.ids_row + i];
    const long long at = (long long)t * a.teacher_row + i;
    says = a.teacher_bf16 ? as_float(reinterpret_cast<const uint16_t *>(a.teacher)[at]) : reinterpret_cast<const float *>(a.teacher)[at];
}
__device__ __forceinline__ bool is_there(const DistillDev &a, int id, float says) { return id >= 0 && uint32_t(id) < a.vocab && says != -INFINITY; }

template <int WARPS>
struct Shared {
    Partial parts[kMaxSplit], warp_part[WARPS];
    Row row;
    float warp_most[WARPS];
    int repeated;
};

// A far row, of which `row` knows the largest logits: its sums once more, and all that is wanted of it, from distances to the largest, which
// are exact to the last bits wherever the logits lie.  A way of its own, because one more operation per logit, or more registers, would
// slow all rows; its loops stay rolled for the same reason (with two vectors at a time the other rows' spill, 458 us instead of 433).
// 4096 x 151936 bfloat16 with all but the named logits at -1e10: 1060 us.
template <typename T, bool GRAD, bool SHORT>
__device__ __forceinline__ void do_far_row(const DistillDev &a, Shared<Shape<GRAD, SHORT>::kWarps> &shared) {
    using Vec = Vector<T>;
    constexpr uint32_t N = Vec::N, kWarps = Shape<GRAD, SHORT>::kWarps, kThreads = 32 * kWarps;
    extern __shared__ __align__(128) char dynamic[];
    const uint32_t part = blockIdx.x % a.split, t = blockIdx.x / a.split, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Span sp = span_of<T>(a, t, part);
    const Named e(dynamic + Shape<GRAD, SHORT>::kRingBytes, a.top);
    const uint8_t *mark = reinterpret_cast<const uint8_t *>(e.marks) - sp.lo;
    const float m = shared.row.m;
    const double base = fmaxf(shared.row.named_m, m > kMasked ? m : -FLT_MAX);
    const float2 minus = make_float2(-m, -m), c2 = make_float2(a.c, a.c);
    if (a.split > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");   // this CTA has read its parts
    // exp(z) of a vector in units of that of m
    auto powers = [&](const uint4 &x, float2 (&v)[N / 2]) {
        Vec::unpack(x, v);
#pragma unroll
        for (int i = 0; i < int(N) / 2; ++i) {
            v[i] = mul2(add2(v[i], minus), c2);
            v[i] = make_float2(exp2_approx(v[i].x), exp2_approx(v[i].y));
        }
    };
    // which elements of a vector are the row's
    auto inside = [&](uint32_t j) {
        uint32_t bits = (1u << N) - 1;
        if (j * N < sp.off) bits &= bits << (sp.off - j * N);
        if ((j + 1) * N > sp.end) bits &= (1u << (sp.end - j * N)) - 1;
        return bits;
    };
    auto load = [&](uint32_t j, uint32_t bits) {
        if (bits == (1u << N) - 1) return reinterpret_cast<const uint4 *>(sp.z)[j];
        alignas(16) T v[N];
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] = bits >> i & 1u ? reinterpret_cast<const T *>(sp.z)[j * N + i] : T(0);
        return *reinterpret_cast<const uint4 *>(v);
    };
    double others = 0.0;
#pragma unroll 1
    for (uint32_t j = sp.lo + threadIdx.x; j < sp.hi; j += kThreads) {
        const uint32_t bits = inside(j);
        float2 v[N / 2];
        powers(Vec::without(load(j, bits), mark[j] | ~bits), v);
#pragma unroll
        for (int w = int(N) / 4; w > 0; w /= 2)
#pragma unroll
            for (int i = 0; i < w; ++i) v[i] = add2(v[i], v[i + w]);
        others += double(v[0].x + v[0].y);
    }
    if (a.kind == GAC_DISTILL_TOP && a.split > 1) {   // the largest value that counts, of all parts: of several with one id the first
        float most = -INFINITY;
        for (uint32_t i = threadIdx.x; i < a.top; i += kThreads) {
            int id, other;
            float says, unsaid;
            read_entry(a, t, i, id, says);
            bool counts = is_there(a, id, says) && says > most;
            for (uint32_t j = 0; j < i && counts; ++j) {
                read_entry(a, t, j, other, unsaid);
                counts = other != id || !is_there(a, other, unsaid);
            }
            if (counts) most = says;
        }
        most = max_lanes(most, 16);
        if (lane == 0) shared.warp_most[warp] = most;
        __syncthreads();
    }
    Partial sum = add_named(a, e, kThreads, max_lanes(shared.warp_most[lane % kWarps], 16), base, 0.0);
    sum.s = float(add_lanes(others, 16));
    sum.m = m;
    sum.named_m = float(base);   // the same in all parts: they are added up as they are
    if (lane == 0) shared.warp_part[warp] = sum;
    __syncthreads();
    if (warp == 0) sum = add_parts(lane < kWarps ? shared.warp_part[lane] : no_part(), a, 32);
    if (a.split > 1) sum = exchange(sum, a, shared.parts, part);
    if (warp == 0) {
        Row r;
        Sums x;
        r.weight = (a.weights ? double(a.weights[t]) : 1.0) * a.inv_temp;
        x.rest = has_rest(sum);
        x.unit = 0.0;
        x.rest_unit = x.rest ? (double(m) - base) * a.inv_temp : 0.0;
        x.f_rest = x.rest ? exp(x.rest_unit) : 0.0;
        x.f_named = 1.0;
        x.s = x.rest ? double(sum.s) : 0.0;
        const double total = sum.named + x.s * x.f_rest;
        r.total = total < double(INFINITY) ? total : double(NAN);
        x.p_rest = what_is_left(sum.mass);
        if (a.kind != GAC_DISTILL_REVERSE) finish_gradient(a, sum, x, r);
        finish_loss(a, sum, x, r);
        if (lane == 0 && a.loss && part == 0) a.loss[t] = float(r.loss);
        if (lane == 0) shared.row = r;
    }
    if (!GRAD) return;
    __syncthreads();
    char *dz = a.dz + (long long)t * a.dz_row - sp.off * sizeof(T);
    const bool aligned = reinterpret_cast<uint64_t>(dz) % 16 == 0;
    const float2 scale = make_float2(shared.row.others, shared.row.others);
#pragma unroll 1
    for (uint32_t j = sp.lo + threadIdx.x; j < sp.hi; j += kThreads) {
        const uint32_t bits = inside(j);
        float2 v[N / 2];
        powers(load(j, bits), v);
#pragma unroll
        for (int i = 0; i < int(N) / 2; ++i) v[i] = mul2(v[i], scale);
        const uint4 y = Vec::pack(v);
        if (aligned && bits == (1u << N) - 1) {
            __stcs(reinterpret_cast<uint4 *>(dz) + j, y);
        } else {
            alignas(16) T w[N];
            *reinterpret_cast<uint4 *>(w) = y;
#pragma unroll
            for (uint32_t i = 0; i < N; ++i)
                if (bits >> i & 1u) reinterpret_cast<T *>(dz)[j * N + i] = w[i];
        }
    }
    __syncthreads();
    put_named<T>(a, e, shared.row, kThreads, dz, base, 1.0);
}

template <typename T, bool GRAD, bool SHORT>
__global__ void __launch_bounds__(Shape<GRAD, SHORT>::kThreads, Shape<GRAD, SHORT>::kCtas)
distill_kernel(const __grid_constant__ DistillDev a) {
    using Vec = Vector<T>;
    using C = Shape<GRAD, SHORT>;
    constexpr int N = Vec::N, kThreads = C::kThreads, kWarps = C::kWarps, kFlight = C::kFlight, kRing = C::kRing;
    extern __shared__ __align__(128) char dynamic[];   // a ring that begins off 32 bytes takes every sector of a row from L2 twice (484 us)
    __shared__ Shared<kWarps> shared;
    Row &row = shared.row;

    const uint32_t part = blockIdx.x % a.split, t = blockIdx.x / a.split;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, top = a.top;
    const Span sp = span_of<T>(a, t, part);
    const uint32_t ring = smem_addr(dynamic) + threadIdx.x * 16;
    const Named e(dynamic + C::kRingBytes, top);
    for (uint32_t i = threadIdx.x; i < a.mark_words; i += kThreads) e.marks[i] = 0;
    if (threadIdx.x == 0) shared.repeated = 0;

    const uint32_t groups = sp.whole_hi > sp.whole_lo ? (sp.whole_hi - sp.whole_lo + kFlight * kThreads - 1) / (kFlight * kThreads) : 0;
    // A thread's own vectors pass through a ring in shared memory, kRing groups of kFlight of them, and no other thread sees them.
    uint64_t first, drop;   // values alone: a row is read once
    if (GRAD) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(first));
    else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(first));
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(drop));
    auto issue = [&](uint32_t group, uint32_t from, uint64_t policy) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const uint32_t j = sp.whole_lo + threadIdx.x + (from * kFlight + u) * kThreads;
            if (from < groups && j < sp.whole_hi)
                asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(ring + ((group % kRing) * kFlight + u) * (kThreads * 16)),
                             "l"(reinterpret_cast<const uint4 *>(sp.z) + j), "l"(policy) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto take = [&](uint32_t group, uint4 (&x)[kFlight]) {   // the oldest group
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[u].x), "=r"(x[u].y), "=r"(x[u].z), "=r"(x[u].w)
                         : "r"(ring + ((group % kRing) * kFlight + u) * (kThreads * 16)) : "memory");
    };
    // elements of a vector that is not whole, by one thread each
    auto edge = [&](auto each) {
        if (threadIdx.x >= 2 * N || sp.lo >= sp.hi) return;
        const uint32_t vector = threadIdx.x < N ? 0 : sp.vectors - 1, place = vector * N + threadIdx.x % N;
        if (vector < sp.lo || vector >= sp.hi || (vector >= sp.whole_lo && vector < sp.whole_hi) || (threadIdx.x >= N && sp.vectors == 1)) return;
        if (place >= sp.off && place < sp.end) each(place);
    };
    const float2 c2 = make_float2(a.c, a.c);
    int id0 = -1;     // the thread's first entry, on its way early
    float l0 = 0.f;
    if (threadIdx.x < top) read_entry(a, t, threadIdx.x, id0, l0);
#pragma unroll
    for (int g = 0; g < kRing; ++g) issue(g, g, first);
    __syncthreads();
    // ---- what the teacher names
    bool any = false;
    float most = -INFINITY, z0 = 0.f;
    for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
        int id = id0;
        float l = l0;
        if (i >= kThreads) read_entry(a, t, i, id, l);
        uint32_t place = kNowhere;
        if (is_there(a, id, l)) {
            any = true;
            most = fmaxf(most, l);
            place = uint32_t(id) + sp.off;
            if (place >= sp.lo * N && place < sp.hi * N) {
                const float z = as_float(reinterpret_cast<const T *>(sp.z)[place]);
                if (i < kThreads) z0 = z;   // not waited for yet
                else e.z[i] = z;
                const uint32_t bit = 1u << ((place / N - sp.lo) % 4 * 8 + place % N);
                if (atomicOr(e.marks + (place / N - sp.lo) / 4, bit) & bit) shared.repeated = 1;
            } else {
                place = kNowhere;
            }
        }
        e.at[i] = place;
        e.l[i] = l;
    }
    most = max_lanes(most, 16);
    if (lane == 0) shared.warp_most[warp] = most;
    any = __syncthreads_or(any);
    if (any && a.split > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");   // this CTA has started
    if (shared.repeated) {   // of several with the same token the first counts
        for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
            const uint32_t at = e.at[i];
            bool seen = false;
            for (uint32_t j = 0; at != kNowhere && j < i; ++j) seen |= e.at[j] == at;
            e.p[i] = seen ? 1.0 : 0.0;
        }
        __syncthreads();
        // p of kind top is told from the largest value that counts.  A CTA with a part of the row does not know what other parts hold: if
        // it drops the largest of all, the row is gone over once more, like a far one
        const float all = max_lanes(shared.warp_most[lane % kWarps], 16);
        most = -INFINITY;
        for (uint32_t i = threadIdx.x; i < top; i += kThreads) {
            if (e.p[i] != 0.0 && e.at[i] != kNowhere) {
                e.at[i] = kNowhere;
                if (e.l[i] >= all) shared.repeated = 2;
            } else if (e.at[i] != kNowhere) {
                most = fmaxf(most, e.l[i]);
            }
        }
        most = max_lanes(most, 16);
        __syncthreads();
        if (a.split == 1 && lane == 0) shared.warp_most[warp] = most;
        __syncthreads();
    }

    float named_level = -FLT_MAX;
    if (any) {
        // ---- largest logit and sum of exponentials of all others
        float m = -FLT_MAX, level = level_of(m, a.c);
        float2 s = make_float2(0.f, 0.f);
        auto raise = [&](float next) {
            const float next_level = level_of(next, a.c), f = exp2_approx(level - next_level);
            s = mul2(s, make_float2(f, f));
            m = next;
            level = next_level;
        };
        auto add = [&](const uint4 &y) {
            float2 v[N / 2];
            Vec::unpack(y, v);
            const float2 minus = make_float2(-level, -level);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                v[i] = fma2(v[i], c2, minus);
                v[i] = make_float2(exp2_approx(v[i].x), exp2_approx(v[i].y));
            }
#pragma unroll
            for (int w = N / 4; w > 0; w /= 2)
#pragma unroll
                for (int i = 0; i < w; ++i) v[i] = add2(v[i], v[i + w]);
            s = add2(s, v[0]);
        };
        const uint8_t *mark = reinterpret_cast<const uint8_t *>(e.marks) - sp.lo;
        for (uint32_t g = 0; g < groups; ++g) {
            uint4 x[kFlight];
            take(g, x);
            issue(g + kRing, g + kRing, first);
            const uint32_t j = sp.whole_lo + threadIdx.x + g * (kFlight * kThreads);
            if (j + (kFlight - 1) * kThreads < sp.whole_hi) {
                uint32_t marked[kFlight], some = 0;
#pragma unroll
                for (int u = 0; u < kFlight; ++u) some |= marked[u] = mark[j + u * kThreads];
                if (some) {
#pragma unroll
                    for (int u = 0; u < kFlight; ++u) x[u] = Vec::without(x[u], marked[u]);
                }
                uint4 big = x[0];
#pragma unroll
                for (int u = 1; u < kFlight; ++u) big = Vec::larger(big, x[u]);
                raise(fmaxf(m, Vec::largest(big)));
#pragma unroll
                for (int u = 0; u < kFlight; ++u) add(x[u]);
            } else {
#pragma unroll
                for (int u = 0; u < kFlight - 1; ++u)
                    if (j + u * kThreads < sp.whole_hi) {
                        const uint4 y = Vec::without(x[u], mark[j + u * kThreads]);
                        raise(fmaxf(m, Vec::largest(y)));
                        add(y);
                    }
            }
        }
        edge([&](uint32_t place) {
            if (reinterpret_cast<const uint8_t *>(e.marks)[place / N - sp.lo] >> (place % N) & 1u) return;
            const float v = as_float(reinterpret_cast<const T *>(sp.z)[place]), next = fmaxf(m, v), next_level = level_of(next, a.c);
            const float f = exp2_approx(level - next_level);
            s = make_float2(s.x * f + exp2_approx(fmaf(v, a.c, -next_level)), s.y * f);
            m = next;
            level = next_level;
        });
        if (GRAD) {   // on its way meanwhile
#pragma unroll
            for (int g = 0; g < kRing; ++g) issue(g, groups - 1 - g, drop);
        }
        most = max_lanes(shared.warp_most[lane % kWarps], 16);
        float m_named = -FLT_MAX;
        for (uint32_t i = threadIdx.x; i < top; i += kThreads)
            if (e.at[i] != kNowhere) {
                if (i < kThreads) e.z[i] = z0;
                m_named = fmaxf(m_named, e.z[i]);
            }
        m_named = max_lanes(m_named, 16);
        named_level = level_of(m_named, a.c);
        Partial mine = add_named(a, e, kThreads, most, 0.0, double(named_level) * M_LN2);
        mine.named_m = m_named;
        mine.m = max_lanes(m, 16);
        mine.s = add_lanes((s.x + s.y) * exp2_approx(level - level_of(mine.m, a.c)), 16);
        if (lane == 0) shared.warp_part[warp] = mine;
        __syncthreads();
        // ---- the row's numbers
        Partial sum;
        if (warp == 0) sum = add_parts(lane < kWarps ? shared.warp_part[lane] : no_part(), a, 32);
        if (a.split > 1) {
            if (a.kind == GAC_DISTILL_TOP && shared.repeated == 2) sum.mass = NAN;
            sum = exchange(sum, a, shared.parts, part);
        }
        Row r;
        Sums more;
        auto tell = [&]() {   // of a far row too, and then once more: a branch here would cost more
            if (warp == 0 && a.loss && part == 0) {
                if (a.kind != GAC_DISTILL_REVERSE) finish_loss(a, sum, more, r);
                if (lane == 0) a.loss[t] = float(r.loss);
            }
        };
        if (warp == 0) {
            r.weight = (a.weights ? double(a.weights[t]) : 1.0) * a.inv_temp;
            r.m = sum.m;
            r.named_m = sum.named_m;
            r.far = far_row(a, sum.m, sum.named_m) || sum.mass != sum.mass;
            more = start(a, sum, r);
            if (a.kind == GAC_DISTILL_REVERSE) finish_loss(a, sum, more, r);
            else finish_gradient(a, sum, more, r);
            if (GRAD && lane == 0) row = r;
        }
        if (!GRAD) {
            tell();
            if (threadIdx.x == 0) {
                row.m = r.m;
                row.named_m = r.named_m;
                row.far = r.far;
            }
        }
        __syncthreads();
        if (row.far) {
            do_far_row<T, GRAD, SHORT>(a, shared);
            asm volatile("cp.async.wait_all;" ::: "memory");
            return;
        }
        if (GRAD) tell();
    } else if (a.loss && part == 0 && threadIdx.x == 0) {
        a.loss[t] = 0.0f;   // nothing to compare with
    }

    // ---- gradient, from the row's end to its beginning: what was read last is in L2 for certain
    if (GRAD) {
        char *dz = a.dz + (long long)t * a.dz_row - sp.off * sizeof(T);   // place 0
        const bool aligned = reinterpret_cast<uint64_t>(dz) % 16 == 0;
        auto put = [&](uint32_t j, const uint4 &y) {   // a whole vector
            if (aligned) {
                __stcs(reinterpret_cast<uint4 *>(dz) + j, y);
            } else {
                const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(dz)[j * N + i] = w[i % 4];
                    else reinterpret_cast<uint16_t *>(dz)[j * N + i] = uint16_t(w[i / 2 % 4] >> (i % 2 * 16));
                }
            }
        };
        if (any) {
            const float others = row.others, level = row.level;
            const float2 minus = make_float2(-level, -level), by = make_float2(others, others);
            auto gradient = [&](const uint4 &y) {
                float2 v[N / 2];
                Vec::unpack(y, v);
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    v[i] = fma2(v[i], c2, minus);
                    v[i] = mul2(make_float2(exp2_approx(v[i].x), exp2_approx(v[i].y)), by);
                }
                return Vec::pack(v);
            };
            for (uint32_t g = 0; g < groups; ++g) {
                uint4 x[kFlight];
                take(g, x);
                issue(g + kRing, groups - 1 - g - kRing, drop);
                const uint32_t j = sp.whole_lo + threadIdx.x + (groups - 1 - g) * (kFlight * kThreads);
                if (aligned && j + (kFlight - 1) * kThreads < sp.whole_hi) {
#pragma unroll
                    for (int u = 0; u < kFlight; ++u) __stcs(reinterpret_cast<uint4 *>(dz) + j + u * kThreads, gradient(x[u]));
                } else {
#pragma unroll
                    for (int u = 0; u < kFlight; ++u)
                        if (j + u * kThreads < sp.whole_hi) put(j + u * kThreads, gradient(x[u]));
                }
            }
            edge([&](uint32_t place) {
                const float v = as_float(reinterpret_cast<const T *>(sp.z)[place]);
                reinterpret_cast<T *>(dz)[place] = from_float(exp2_approx(fmaf(v, a.c, -level)) * others, T{});
            });
        } else {
            for (uint32_t j = sp.whole_lo + threadIdx.x; j < sp.whole_hi; j += kThreads) put(j, make_uint4(0, 0, 0, 0));
            edge([&](uint32_t place) { reinterpret_cast<T *>(dz)[place] = T(0); });
        }
        if (any) {
            __syncthreads();   // the named tokens' own gradients over what has been written
            put_named<T>(a, e, row, kThreads, dz, 0.0, power_of_two(named_level - row.unit));
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");   // of a row without entries the first loads may still be on their way
}

struct Launch {
    void (*kernel)(const DistillDev);
    uint32_t threads, ctas;
    size_t ring;
};
template <typename T, bool GRAD, bool SHORT>
Launch launch_with() {
    using C = Shape<GRAD, SHORT>;
    return {distill_kernel<T, GRAD, SHORT>, C::kThreads, C::kCtas, C::kRingBytes};
}
template <typename T>
Launch launch_for(bool grad, bool brief) {
    return grad ? (brief ? launch_with<T, true, true>() : launch_with<T, true, false>()) : (brief ? launch_with<T, false, true>() : launch_with<T, false, false>());
}
Launch launch_of(bool bf16, bool grad, bool brief) { return bf16 ? launch_for<uint16_t>(grad, brief) : launch_for<float>(grad, brief); }

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
    if (a.vocab < 1 || a.vocab > GAC_DISTILL_MAX_ROW_BYTES / (a.dtype == GAC_BF16 ? 2 : 4))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "vocab must be at least 1, and its logits of a row at most %s%lld bytes", "", (long long)GAC_DISTILL_MAX_ROW_BYTES);
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
    d.c_off = (M_LOG2E / a.temperature - double(d.c)) * M_LN2;
    const uint32_t vec = 16 / uint32_t(size), vectors = (a.vocab + 2 * vec - 2) / vec;   // at most, wherever a row starts
    const bool grad = a.d_logits != nullptr;
    const uint64_t row = uint64_t(a.vocab) * size;
    const bool brief = row <= (grad ? kInUse / (148 * Shape<true, true>::kCtas) : 256u << 10);   // short rows
    const Launch shape = launch_of(a.dtype == GAC_BF16, grad, brief);
    // Parts of a row: what takes least, by 44 bytes a nanosecond and SM, and by the chain from a row's last load to its first gradient
    // (5 us, with the gradient 8, where parts wait for each other 1.5 more).  With the gradient so many that the rows in use
    // at once stay in L2 between the two passes (4096 rows of 304 kB: 499 us with one part, 434 with two; 8191 rows of 128 kB, which
    // fit whole: 310 and 353).
    d.split = 1;
    double least = INFINITY;
    for (uint32_t split = 1; split <= kMaxSplit; split *= 2) {
        const bool fits = !grad || uint64_t(148 * shape.ctas / split) * row <= kInUse || uint64_t(a.n_tokens) * row <= kInUse;
        if (!fits && split < kMaxSplit) continue;
        const uint64_t per_sm = (uint64_t(a.n_tokens) * split + 147) / 148, waves = (per_sm + shape.ctas - 1) / shape.ctas;
        const double time = double(per_sm) * double(row * (grad ? 2 : 1)) / split / 44.0 + double(waves) * ((grad ? 8000.0 : 5000.0) + (split > 1 ? 1500.0 : 0.0));
        if (time < least) {
            least = time;
            d.split = split;
        }
    }
    d.mark_words = ((vectors + d.split - 1) / d.split + 3) / 4;
    const size_t smem = shape.ring + size_t(a.top) * 28 + size_t(d.mark_words) * 4;
    Range range("gac_distill");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    static std::atomic<bool> allowed[8][64];   // once for each device
    std::atomic<bool> *done = cuda_device >= 0 && cuda_device < 64 ? &allowed[(a.dtype == GAC_BF16) + 2 * grad + 4 * brief][cuda_device] : nullptr;
    if (!done || !*done) {
        GAC_CUDA(nullptr, cudaFuncSetAttribute(shape.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMaxSmem)));
        if (done) *done = true;
    }
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3(a.n_tokens * d.split);
    how.blockDim = dim3(shape.threads);
    how.dynamicSmemBytes = smem;
    how.stream = static_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = d.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    how.attrs = attr;
    how.numAttrs = 1;
    GAC_CUDA(nullptr, cudaLaunchKernelEx(&how, shape.kernel, d));
    return GAC_OK;
}

}  // extern "C"
