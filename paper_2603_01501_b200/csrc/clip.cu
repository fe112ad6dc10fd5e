// Global gradient norm over a list of tensors, and clipping (gac_clip_* of include/gac.h).
//
//   norm = sqrt(sum g_i^2),   out_i = min(1, max_norm / (norm + eps)) g_i
//
// The norm has to be known before the first element can be written, so a list beyond the chip's
// memory is read twice and written once: the floor is the HBM traffic of that.  Squares are summed in
// binary64 (a product of two binary32 values is exact there, and no scale of the gradient overflows or
// vanishes), in a fixed order: chunk c belongs to CTA c mod grid, each CTA leaves one partial sum, and they are
// added in index order.  One cooperative launch does both passes; the CTAs meet in between.
// Measured: 1.5 B float32 elements 2.78 ms = 6.66 TB/s over the three passes (1.03 of a plain copy's rate), 0.25 B
// bfloat16 240 us = 6.2 TB/s (its first pass converts every element to binary64 and is held up by that), 2^20 float32
// 8.2 us and the 38 tensors of a small mixed list 6.2 us, which are one launch and one meeting of all CTAs.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <cstddef>
#include <map>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "gac.h"
#include "gac_host.h"

static_assert(sizeof(gac_clip_tensor) == 32 && sizeof(gac_clip_result) == 32, "clip structs layout");

namespace {

constexpr int kThreads = 256;
constexpr int kChunkElems = 16384, kShortChunkElems = 4096;
constexpr uint64_t kShortList = 1ull << 21;   // elements
constexpr int kCtasPerSm = 4;
constexpr int kSumFlight = 8;     // vectors of 16 bytes in flight per thread, first pass
constexpr int kApplyFlight = 4;   // second pass
constexpr uint32_t kBf16 = 1u, kInPlace = 2u;

struct __align__(16) ClipChunk {
    uint64_t g, out;   // device addresses of the chunk's first element
    uint32_t n, flags;
    uint64_t pad;
};
static_assert(sizeof(ClipChunk) == 32, "chunk descriptors are read as two 16-byte words");

__device__ __forceinline__ ClipChunk load_chunk(const ClipChunk *table, uint32_t c) {
    const uint4 *p = reinterpret_cast<const uint4 *>(table + c);
    const uint4 a = __ldg(p), b = __ldg(p + 1);
    ClipChunk ch;
    ch.g = (uint64_t(a.y) << 32) | a.x;
    ch.out = (uint64_t(a.w) << 32) | a.z;
    ch.n = b.x;
    ch.flags = b.y;
    ch.pad = 0;
    return ch;
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// One element of either type at index i.
__device__ __forceinline__ float load_one(uint64_t base, uint32_t i, bool bf16) {
    return bf16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t *>(base)[i]) << 16)
                : reinterpret_cast<const float *>(base)[i];
}
__device__ __forceinline__ void store_one(uint64_t base, uint32_t i, bool bf16, float v) {
    if (bf16) reinterpret_cast<uint16_t *>(base)[i] = uint16_t(pack_bf16x2(v, 0.0f) & 0xFFFFu);
    else reinterpret_cast<float *>(base)[i] = v;
}

// Elements before the first 16-byte boundary of the chunk's input.
__device__ __forceinline__ uint32_t head_elems(uint64_t base, uint32_t n, bool bf16) {
    const uint32_t off = uint32_t((16u - (base & 15u)) & 15u) >> (bf16 ? 1 : 2);
    return off < n ? off : n;
}

__device__ __forceinline__ void add_square(double &acc, float x) {
    const double v = double(x);
    acc = __fma_rn(v, v, acc);
}

__device__ __forceinline__ void add_squares(double (&acc)[2], uint4 w, bool bf16) {
    if (bf16) {
        add_square(acc[0], lo_bf16(w.x)); add_square(acc[1], hi_bf16(w.x));
        add_square(acc[0], lo_bf16(w.y)); add_square(acc[1], hi_bf16(w.y));
        add_square(acc[0], lo_bf16(w.z)); add_square(acc[1], hi_bf16(w.z));
        add_square(acc[0], lo_bf16(w.w)); add_square(acc[1], hi_bf16(w.w));
    } else {
        add_square(acc[0], __uint_as_float(w.x)); add_square(acc[1], __uint_as_float(w.y));
        add_square(acc[0], __uint_as_float(w.z)); add_square(acc[1], __uint_as_float(w.w));
    }
}

__device__ double cta_sum(double v, double *shared) {
    for (int o = 16; o > 0; o >>= 1) v = __dadd_rn(v, __shfl_down_sync(0xFFFFFFFFu, v, o));
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) shared[warp] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kThreads / 32; ++w) s = __dadd_rn(s, shared[w]);
    __syncthreads();
    return s;   // valid in thread 0
}

__device__ __forceinline__ uint4 scaled(uint4 w, float s, bool bf16) {
    if (bf16)
        return make_uint4(pack_bf16x2(lo_bf16(w.x) * s, hi_bf16(w.x) * s), pack_bf16x2(lo_bf16(w.y) * s, hi_bf16(w.y) * s),
                          pack_bf16x2(lo_bf16(w.z) * s, hi_bf16(w.z) * s), pack_bf16x2(lo_bf16(w.w) * s, hi_bf16(w.w) * s));
    return make_uint4(__float_as_uint(__uint_as_float(w.x) * s), __float_as_uint(__uint_as_float(w.y) * s),
                      __float_as_uint(__uint_as_float(w.z) * s), __float_as_uint(__uint_as_float(w.w) * s));
}

// This CTA's share of the sum of squares (valid in thread 0).
__device__ double chunk_squares(const ClipChunk *__restrict__ table, uint32_t n_chunks, double *shared) {
    double acc[2] = {0.0, 0.0};
    for (uint32_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const ClipChunk ch = load_chunk(table, c);
        const bool bf16 = ch.flags & kBf16;
        const uint32_t head = head_elems(ch.g, ch.n, bf16);
        const uint32_t per = bf16 ? 8u : 4u, vecs = (ch.n - head) / per;
        const uint4 *v = reinterpret_cast<const uint4 *>(ch.g + uint64_t(head) * (bf16 ? 2 : 4));
        if (threadIdx.x < head) add_square(acc[0], load_one(ch.g, threadIdx.x, bf16));
        uint32_t i = threadIdx.x;
        for (; i + (kSumFlight - 1) * kThreads < vecs; i += kSumFlight * kThreads) {
            uint4 w[kSumFlight];
#pragma unroll
            for (int u = 0; u < kSumFlight; ++u) w[u] = v[i + u * kThreads];
#pragma unroll
            for (int u = 0; u < kSumFlight; ++u) add_squares(acc, w[u], bf16);
        }
        for (; i < vecs; i += kThreads) add_squares(acc, v[i], bf16);
        for (uint32_t j = head + vecs * per + threadIdx.x; j < ch.n; j += kThreads)
            add_square(acc[0], load_one(ch.g, j, bf16));
    }
    return cta_sum(__dadd_rn(acc[0], acc[1]), shared);
}

// The CTAs' shares in index order, by any CTA (valid in thread 0).
__device__ double all_squares(const double *partials, double *shared) {
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kThreads) s = __dadd_rn(s, __ldcg(partials + i));
    return cta_sum(s, shared);
}

// Waits until every CTA of a cooperative launch has arrived.  They are all resident, so this ends by itself; the limit only
// keeps a mistake from holding the GPU.  Arrivals and giving up are bits of one word, so that all CTAs come to the
// same end: once the last has arrived nobody can give up any more, and once one has given up nobody goes on.  Called by
// one thread of each CTA.
constexpr unsigned long long kGaveUp = 1ull << 63;
__device__ bool meet(unsigned long long *arrived, unsigned long long limit_ns) {
    __threadfence();
    if (limit_ns == 0) atomicOr(arrived, kGaveUp);   // not even for those that are nearly there; this one has not arrived yet
    const unsigned long long old = atomicAdd(arrived, 1ull), target = (old / gridDim.x + 1) * gridDim.x;
    if (old & kGaveUp) return false;   // another CTA did, or an earlier call that nobody has been told of yet
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    bool late = false;
    for (uint32_t i = 0;; ++i) {
        unsigned long long now;
        asm volatile("ld.acquire.gpu.u64 %0, [%1];" : "=l"(now) : "l"(arrived) : "memory");
        if (now & kGaveUp) return false;
        if (now >= target) return true;
        if (!late && i % 1024 == 0) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            late = t - t0 >= limit_ns || i >= (1u << 28);
        }
        if (late && atomicCAS(arrived, now, now | kGaveUp) == now) return false;   // fails only where another CTA arrives
    }
}

enum { kSumOnly = 0, kApplyOnly = 1, kBoth = 2 };

// kBoth: one cooperative launch.  The second pass walks the chunks backwards: the last ones read are still in the L2 cache
// (126 MB), and the stores are marked to leave it first.
template <int MODE>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
clip_kernel(const ClipChunk *__restrict__ table, uint32_t n_chunks, double *partials, unsigned long long *arrived,
            unsigned long long limit_ns, double *sumsq, double max_norm, double eps, float *norm_out, gac_clip_result *rec) {
    __shared__ double shared[kThreads / 32];
    __shared__ float factor;
    __shared__ int state;   // 0 as it should be, 1 not finite, 2 a wait ran out; kSumOnly: 1 in the last CTA
    if (MODE != kApplyOnly) {
        const double mine = chunk_squares(table, n_chunks, shared);
        if (MODE == kSumOnly) {
            if (threadIdx.x == 0) {
                partials[blockIdx.x] = mine;
                __threadfence();
                state = ((atomicAdd(arrived, 1ull) + 1) & ~kGaveUp) % gridDim.x == 0;
            }
            __syncthreads();
            if (!state) return;
            __threadfence();
            const double s = all_squares(partials, shared);
            if (threadIdx.x == 0) *sumsq = s;
            return;
        }
        if (threadIdx.x == 0) {
            partials[blockIdx.x] = mine;
            state = meet(arrived, limit_ns) ? 0 : 2;
        }
    } else if (threadIdx.x == 0) {
        state = (__ldcg(arrived) & kGaveUp) ? 2 : 0;
    }
    __syncthreads();
    if (state == 2) {   // in every CTA
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            rec->sumsq = rec->norm = rec->scale = __longlong_as_double(0x7FF8000000000000ll);
            rec->timed_out = 1;   // the host clears it once it has read it
            if (norm_out) *norm_out = __int_as_float(0x7FC00000);
        }
        return;
    }
    double s2 = 0.0;
    if (MODE == kBoth) s2 = all_squares(partials, shared);
    else __syncthreads();   // state has been read
    if (threadIdx.x == 0) {
        if (MODE == kApplyOnly) s2 = *sumsq;
        const double norm = __dsqrt_rn(s2), f = __ddiv_rn(max_norm, __dadd_rn(norm, eps));
        const bool bad = !(s2 <= 1.7976931348623157e308);   // NaN or +Inf
        factor = (f < 1.0) ? __double2float_rn(f) : 1.0f;
        state = bad;
        if (blockIdx.x == 0) {
            rec->sumsq = s2;
            rec->norm = norm;
            rec->scale = bad ? 1.0 : double(factor);
            rec->nonfinite = bad;
            if (norm_out) *norm_out = __double2float_rn(norm);
        }
    }
    __syncthreads();
    if (state) return;
    const float s = factor;
    for (uint32_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const ClipChunk ch = load_chunk(table, n_chunks - 1 - c);
        const bool bf16 = ch.flags & kBf16;
        if (s == 1.0f && (ch.flags & kInPlace)) continue;
        const uint32_t size = bf16 ? 2u : 4u;
        uint32_t head = head_elems(ch.g, ch.n, bf16);
        const uint32_t per = 16u / size;
        uint32_t vecs = (ch.n - head) / per;
        if ((ch.g ^ ch.out) & 15u) head = vecs = 0;   // input and output never share a 16-byte boundary
        const uint4 *v = reinterpret_cast<const uint4 *>(ch.g + uint64_t(head) * size);
        uint4 *o = reinterpret_cast<uint4 *>(ch.out + uint64_t(head) * size);
        if (threadIdx.x < head) store_one(ch.out, threadIdx.x, bf16, load_one(ch.g, threadIdx.x, bf16) * s);
        // All warps load, then all warps store: reads and writes reach DRAM in bursts instead of an even mix.  List of
        // 1.5 B float32 elements: 2.91 ms without the barriers and 8 vectors in flight, 2.82 with the first, 2.78 with both.
        for (uint32_t b = 0; b < vecs; b += kApplyFlight * kThreads) {
            uint4 w[kApplyFlight];
#pragma unroll
            for (int u = 0; u < kApplyFlight; ++u)
                if (b + threadIdx.x + u * kThreads < vecs) w[u] = v[b + threadIdx.x + u * kThreads];
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kApplyFlight; ++u)
                if (b + threadIdx.x + u * kThreads < vecs) __stcs(o + b + threadIdx.x + u * kThreads, scaled(w[u], s, bf16));
            __syncthreads();
        }
        for (uint32_t j = head + vecs * per + threadIdx.x; j < ch.n; j += kThreads)
            store_one(ch.out, j, bf16, load_one(ch.g, j, bf16) * s);
    }
}

// New addresses for the chunks of up to kMovedTensors tensors, one to a CTA; they travel as an argument of the launch, so
// nothing on the host has to outlive the call.
constexpr uint32_t kMovedTensors = 512;
struct MovedTensor {
    uint64_t g, out;
    uint32_t first, chunks;   // of the table
};
struct Moved {
    uint32_t chunk_elems, n;
    MovedTensor t[kMovedTensors];
};
__global__ void __launch_bounds__(kThreads) clip_move_kernel(const __grid_constant__ Moved m, ClipChunk *table) {
    const MovedTensor &t = m.t[blockIdx.x];
    for (uint32_t i = threadIdx.x; i < t.chunks; i += kThreads) {
        ClipChunk &c = table[t.first + i];
        const uint64_t off = uint64_t(i) * m.chunk_elems * (c.flags & kBf16 ? 2 : 4);
        c.g = t.g + off;
        c.out = t.out + off;
        c.flags = (c.flags & kBf16) | (t.g == t.out ? kInPlace : 0u);
    }
}

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

}  // namespace

struct gac_clip_ctx {
    int device = 0, sms = 0;
    uint32_t n_chunks = 0;
    uint32_t grid = 0;
    ClipChunk *d_chunks = nullptr;     // the allocation; what follows lies behind the table
    double *d_partials = nullptr;      // one per CTA
    unsigned long long *d_arrived = nullptr;   // CTAs so far, over all calls
    gac_clip_result *d_rec = nullptr;
    gac_clip_result *h_rec = nullptr;  // pinned, from the first call that asks for a record on
    unsigned long long limit_ns = 1000000000ull;
    uint32_t chunk_elems = 0;
    std::vector<std::pair<uint64_t, int32_t>> shape;   // elements and type of every tensor
};

namespace {

void release(gac_clip_ctx *c) {
    if (c->d_chunks) cudaFree(c->d_chunks);   // and all that lies behind the table
    if (c->h_rec) cudaFreeHost(c->h_rec);
}

int check_list(const gac_clip_tensor *list, uint32_t n) {
    std::vector<std::pair<uint64_t, uint64_t>> writes, reads;
    for (uint32_t i = 0; i < n; ++i) {
        const gac_clip_tensor &t = list[i];
        if (t.dtype != GAC_F32 && t.dtype != GAC_BF16)
            return fail(nullptr, GAC_ERR_DTYPE, "tensor %s%lld: gradients are float32 or bfloat16", "", i);
        if (t.reserved != 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "tensor %s%lld: reserved field must be 0", "", i);
        if (t.numel == 0) continue;
        const uint64_t size = t.dtype == GAC_BF16 ? 2 : 4;
        const uint64_t g = reinterpret_cast<uint64_t>(t.g), o = reinterpret_cast<uint64_t>(t.out);
        if (!g || !o) return fail(nullptr, GAC_ERR_INVALID_ARG, "tensor %s%lld has a NULL pointer", "", i);
        if (t.numel > (1ull << 40))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "tensor %s%lld is larger than 2^40 elements", "", i);
        if (g % size || o % size) return fail(nullptr, GAC_ERR_INVALID_ARG, "tensor %s%lld is not element-aligned", "", i);
        writes.emplace_back(o, o + t.numel * size);
        if (g != o) reads.emplace_back(g, g + t.numel * size);
    }
    // what is written must not overlap anything else that is written, nor anything read from elsewhere
    std::sort(writes.begin(), writes.end());
    for (size_t i = 1; i < writes.size(); ++i)
        if (writes[i].first < writes[i - 1].second)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "output buffers of different tensors overlap%s");
    for (const auto &r : reads) {
        auto it = std::lower_bound(writes.begin(), writes.end(), std::make_pair(r.first, uint64_t(0)));
        if ((it != writes.end() && it->first < r.second) || (it != writes.begin() && std::prev(it)->second > r.first))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "an output buffer overlaps a gradient other than its own%s");
    }
    return GAC_OK;
}

// A stream of the library's own, which waits for nobody else's work; one per device, made once (making one takes 100 us).
int setup_stream(int device, cudaStream_t *out) {
    static std::mutex guard;
    static std::map<int, cudaStream_t> streams;
    std::lock_guard<std::mutex> lock(guard);
    cudaStream_t &s = streams[device];
    if (!s) GAC_CUDA(nullptr, cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking));
    *out = s;
    return GAC_OK;
}

int setup(gac_clip_ctx *c, const gac_clip_tensor *list, uint32_t n) {
    GAC_CUDA(nullptr, cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, c->device));
    uint64_t total = 0;
    for (uint32_t i = 0; i < n; ++i) total += list[i].numel;
    // Short lists are cut finer, so that a CTA's turn is short.  Finer against coarser: 0.2 M elements in 15 tensors 6.2 us
    // and 8.2, 2^21 in one 8.5 and 9.3, 2^22 12.4 and 10.3, 0.25 B bfloat16 345 and 240.
    const uint64_t ce = total <= kShortList ? kShortChunkElems : kChunkElems;
    c->chunk_elems = uint32_t(ce);
    std::vector<ClipChunk> table;
    for (uint32_t i = 0; i < n; ++i) {
        const gac_clip_tensor &t = list[i];
        const uint64_t size = t.dtype == GAC_BF16 ? 2 : 4;
        c->shape.emplace_back(t.numel, t.dtype);
        for (uint64_t off = 0; off < t.numel; off += ce) {
            ClipChunk ch;
            ch.g = reinterpret_cast<uint64_t>(t.g) + off * size;
            ch.out = reinterpret_cast<uint64_t>(t.out) + off * size;
            ch.n = uint32_t(std::min<uint64_t>(ce, t.numel - off));
            ch.flags = (t.dtype == GAC_BF16 ? kBf16 : 0u) | (t.g == t.out ? kInPlace : 0u);
            ch.pad = 0;
            table.push_back(ch);
        }
    }
    if (table.size() > 0xFFFFFFF0ull) return fail(nullptr, GAC_ERR_INVALID_ARG, "too many chunks%s");
    c->n_chunks = uint32_t(table.size());
    int resident = 0;   // all CTAs have to be resident at once: they meet between the two passes
    GAC_CUDA(nullptr, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, clip_kernel<kBoth>, kThreads, 0));
    resident = std::max(1, std::min(resident, kCtasPerSm));
    c->grid = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>(uint64_t(c->sms) * resident, table.size())));
    // One block of memory: the table, and behind it, from zeros, partial sums, record and counter.  The call does not return
    // before it is all there: the first launch may be on a stream that nothing else orders behind this call.
    const size_t partials = (size_t(c->grid) + 1) * sizeof(double), chunks = table.size() * sizeof(ClipChunk);
    const size_t behind = partials + sizeof(gac_clip_result) + sizeof(*c->d_arrived);
    table.resize(table.size() + (behind + sizeof(ClipChunk) - 1) / sizeof(ClipChunk));
    cudaStream_t own;
    if (int rc = setup_stream(c->device, &own)) return rc;
    GAC_CUDA(nullptr, cudaMalloc(&c->d_chunks, table.size() * sizeof(ClipChunk)));
    char *base = reinterpret_cast<char *>(c->d_chunks);
    c->d_partials = reinterpret_cast<double *>(base + chunks);
    c->d_rec = reinterpret_cast<gac_clip_result *>(base + chunks + partials);
    c->d_arrived = reinterpret_cast<unsigned long long *>(c->d_rec + 1);
    GAC_CUDA(nullptr, cudaMemcpyAsync(base, table.data(), table.size() * sizeof(ClipChunk), cudaMemcpyHostToDevice, own));
    GAC_CUDA(nullptr, cudaStreamSynchronize(own));
    return GAC_OK;
}

int read_record(gac_clip_ctx *c, cudaStream_t s, gac_clip_result *host_out) {
    if (!host_out) return GAC_OK;
    if (!c->h_rec) GAC_CUDA(nullptr, cudaMallocHost(&c->h_rec, sizeof(gac_clip_result)));   // page-locking takes longer than all of gac_clip_init
    GAC_CUDA(nullptr, cudaMemcpyAsync(c->h_rec, c->d_rec, sizeof(gac_clip_result), cudaMemcpyDeviceToHost, s));
    GAC_CUDA(nullptr, cudaStreamSynchronize(s));
    *host_out = *c->h_rec;
    if (host_out->timed_out) {
        GAC_CUDA(nullptr, cudaMemsetAsync(c->d_arrived, 0, sizeof(*c->d_arrived), s));
        GAC_CUDA(nullptr, cudaMemsetAsync(c->d_rec, 0, sizeof(*c->d_rec), s));
        return fail(nullptr, GAC_ERR_TIMEOUT, "a wait inside the clipping kernel ran out%s");
    }
    if (host_out->nonfinite) return fail(nullptr, GAC_ERR_NONFINITE, "NaN or Inf met in the gradient norm%s");
    return GAC_OK;
}

int check_limits(double max_norm, double eps, const float *norm_out) {
    if (!(max_norm > 0.0)) return fail(nullptr, GAC_ERR_INVALID_ARG, "max_norm must be > 0%s");
    if (!(eps >= 0.0) || !isfinite(eps)) return fail(nullptr, GAC_ERR_INVALID_ARG, "eps must be finite and >= 0%s");
    if (reinterpret_cast<uint64_t>(norm_out) % 4) return fail(nullptr, GAC_ERR_INVALID_ARG, "norm_out must be 4-byte aligned%s");
    return GAC_OK;
}

}  // namespace

extern "C" {

int gac_clip_init(gac_clip_ctx **out, const gac_clip_tensor *list, uint32_t n, int cuda_device) {
    if (!out) return fail(nullptr, GAC_ERR_INVALID_ARG, "out is NULL%s");
    *out = nullptr;
    if (!list || n == 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "empty tensor list%s");
    gac_clip_ctx *c = nullptr;
    try {
        if (int rc = check_list(list, n)) return rc;
        int n_dev = 0;
        if (cudaGetDeviceCount(&n_dev) != cudaSuccess || n_dev == 0)
            return fail(nullptr, GAC_ERR_CUDA, "no CUDA device is available%s");
        if (cuda_device < 0 || cuda_device >= n_dev)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "cuda_device %s%lld out of range", "", cuda_device);
        DeviceGuard guard(cuda_device);
        if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
        c = new gac_clip_ctx;
        c->device = cuda_device;
        if (int rc = setup(c, list, n)) {
            release(c);
            delete c;
            return rc;
        }
    } catch (...) {   // nothing may be thrown through the C boundary
        if (c) {
            release(c);
            delete c;
        }
        return fail(nullptr, GAC_ERR_INVALID_ARG, "out of host memory%s");
    }
    *out = c;
    return GAC_OK;
}

int gac_clip_rebind(gac_clip_ctx *ctx, const gac_clip_tensor *list, uint32_t n, void *cuda_stream) {
    if (!ctx) return fail(nullptr, GAC_ERR_INVALID_ARG, "ctx is NULL%s");
    if (!list || n != ctx->shape.size())
        return fail(nullptr, GAC_ERR_INVALID_ARG, "gac_clip_rebind needs one entry per tensor of the context%s");
    for (uint32_t i = 0; i < n; ++i)
        if (list[i].numel != ctx->shape[i].first || list[i].dtype != ctx->shape[i].second)
            return fail(nullptr, GAC_ERR_INVALID_ARG, "tensor %s%lld changed its size or type; create a new context", "", i);
    try {
        if (int rc = check_list(list, n)) return rc;
    } catch (...) {   // nothing may be thrown through the C boundary
        return fail(nullptr, GAC_ERR_INVALID_ARG, "out of host memory%s");
    }
    Range range("gac_clip_rebind");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    Moved m;
    m.chunk_elems = ctx->chunk_elems;
    m.n = 0;
    uint32_t first = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const uint32_t chunks = uint32_t((list[i].numel + m.chunk_elems - 1) / m.chunk_elems);
        if (chunks)
            m.t[m.n++] = MovedTensor{reinterpret_cast<uint64_t>(list[i].g), reinterpret_cast<uint64_t>(list[i].out), first, chunks};
        first += chunks;
        if (m.n == kMovedTensors || (i + 1 == n && m.n)) {
            clip_move_kernel<<<m.n, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(m, ctx->d_chunks);
            GAC_CUDA(nullptr, cudaGetLastError());
            m.n = 0;
        }
    }
    return GAC_OK;
}

int gac_clip_sumsq(gac_clip_ctx *ctx, void *cuda_stream, double *sumsq_out) {
    if (!ctx) return fail(nullptr, GAC_ERR_INVALID_ARG, "ctx is NULL%s");
    if (!sumsq_out || reinterpret_cast<uint64_t>(sumsq_out) % 8)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "sumsq_out must be an 8-byte aligned device pointer%s");
    Range range("gac_clip_sumsq");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    clip_kernel<kSumOnly><<<ctx->grid, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        ctx->d_chunks, ctx->n_chunks, ctx->d_partials, ctx->d_arrived, ctx->limit_ns, sumsq_out, 0.0, 0.0, nullptr, ctx->d_rec);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

int gac_clip_apply(gac_clip_ctx *ctx, void *cuda_stream, const double *sumsq_in, double max_norm, double eps, float *norm_out,
                   gac_clip_result *host_out) {
    if (!ctx) return fail(nullptr, GAC_ERR_INVALID_ARG, "ctx is NULL%s");
    if (!sumsq_in || reinterpret_cast<uint64_t>(sumsq_in) % 8)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "sumsq_in must be an 8-byte aligned device pointer%s");
    if (int rc = check_limits(max_norm, eps, norm_out)) return rc;
    Range range("gac_clip_apply");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    clip_kernel<kApplyOnly><<<ctx->grid, kThreads, 0, s>>>(ctx->d_chunks, ctx->n_chunks, ctx->d_partials, ctx->d_arrived, ctx->limit_ns,
                                                           const_cast<double *>(sumsq_in), max_norm, eps, norm_out, ctx->d_rec);
    GAC_CUDA(nullptr, cudaGetLastError());
    return read_record(ctx, s, host_out);
}

int gac_clip_grad_norm(gac_clip_ctx *ctx, void *cuda_stream, double max_norm, double eps, float *norm_out,
                       gac_clip_result *host_out) {
    if (!ctx) return fail(nullptr, GAC_ERR_INVALID_ARG, "ctx is NULL%s");
    if (int rc = check_limits(max_norm, eps, norm_out)) return rc;
    Range range("gac_clip_grad_norm");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    double *none = nullptr;
    void *args[] = {&ctx->d_chunks, &ctx->n_chunks, &ctx->d_partials, &ctx->d_arrived, &ctx->limit_ns, &none, &max_norm, &eps, &norm_out, &ctx->d_rec};
    GAC_CUDA(nullptr, cudaLaunchCooperativeKernel(reinterpret_cast<const void *>(&clip_kernel<kBoth>), dim3(ctx->grid), dim3(kThreads), args, 0, s));
    return read_record(ctx, s, host_out);
}

int gac_clip_set_timeout(gac_clip_ctx *ctx, uint32_t timeout_ms) {
    if (!ctx) return fail(nullptr, GAC_ERR_INVALID_ARG, "ctx is NULL%s");
    ctx->limit_ns = 1000000ull * timeout_ms;
    return GAC_OK;
}

int gac_clip_free(gac_clip_ctx *ctx) {
    if (!ctx) return GAC_OK;
    {
        DeviceGuard guard(ctx->device);
        release(ctx);
    }
    delete ctx;
    return GAC_OK;
}

}  // extern "C"
