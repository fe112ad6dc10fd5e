// Causal attention over a pack of sequences, grouped heads, forward and backward (gac_attn_* of include/gac.h).
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <cstddef>

#include "gac.h"
#include "gac_host.h"
#include "attention_kernels.cuh"

namespace {

constexpr int kWarps = 4;

struct HeadsDev {
    char *p;
    long long token, head;   // bytes
};
struct PlainDev {
    HeadsDev q, k, v, o, d_o, d_q, d_k, d_v;
    float *lse, *delta;
    const int32_t *cu;
    uint32_t n_tokens, n_seqs, q_heads, kv_heads, head_dim;
    float scale;
};

// Start and end of the sequence of token t; an empty range for a token that belongs to none.
__device__ bool sequence_of(const PlainDev &a, uint32_t t, uint32_t *first, uint32_t *end) {
    uint32_t lo = 0, hi = a.n_seqs;
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (uint32_t(max(a.cu[mid], 0)) <= t) lo = mid;
        else hi = mid - 1;
    }
    if (lo == a.n_seqs) return false;
    *first = lo ? uint32_t(max(a.cu[lo], 0)) : 0u;
    *end = min(uint32_t(max(a.cu[lo + 1], 0)), a.n_tokens);
    return t < *end;
}

// Four elements of a row, elements lane*4 .. +3 (zero beyond head_dim).
__device__ float4 row4(const HeadsDev &h, uint32_t t, uint32_t head, uint32_t dim) {
    const uint32_t lane = threadIdx.x & 31;
    if (lane * 4 >= dim) return make_float4(0.f, 0.f, 0.f, 0.f);
    const uint2 w = *reinterpret_cast<const uint2 *>(h.p + (long long)t * h.token + (long long)head * h.head + lane * 8);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u));
}
__device__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ void put4(const HeadsDev &h, uint32_t t, uint32_t head, uint32_t dim, float4 v) {
    const uint32_t lane = threadIdx.x & 31;
    if (lane * 4 >= dim) return;
    *reinterpret_cast<uint2 *>(h.p + (long long)t * h.token + (long long)head * h.head + lane * 8) =
        make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}
__device__ float dot4(float4 a, float4 b) {
    float s = a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w;
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}
__device__ void add4(float4 &a, float s, float4 b) {
    a.x += s * b.x;
    a.y += s * b.y;
    a.z += s * b.z;
    a.w += s * b.w;
}

__global__ void attn_delta_kernel(const __grid_constant__ PlainDev a) {
    const uint32_t h = blockIdx.y, t = blockIdx.x * kWarps + threadIdx.x / 32;
    if (t >= a.n_tokens) return;
    const float d = dot4(row4(a.o, t, h, a.head_dim), row4(a.d_o, t, h, a.head_dim));
    if ((threadIdx.x & 31) == 0) a.delta[size_t(h) * a.n_tokens + t] = d;
}

__global__ void attn_dq_kernel(const __grid_constant__ PlainDev a) {
    const uint32_t h = blockIdx.y, t = blockIdx.x * kWarps + threadIdx.x / 32;
    if (t >= a.n_tokens) return;
    const uint32_t kv = h / (a.q_heads / a.kv_heads);
    uint32_t first, end;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (sequence_of(a, t, &first, &end)) {
        const float4 q = row4(a.q, t, h, a.head_dim), g = row4(a.d_o, t, h, a.head_dim);
        const float lse = a.lse[size_t(h) * a.n_tokens + t], delta = a.delta[size_t(h) * a.n_tokens + t];
        for (uint32_t j = first; j <= t; ++j) {
            const float4 k = row4(a.k, j, kv, a.head_dim);
            const float p = expf(dot4(q, k) * a.scale - lse);
            add4(acc, p * (dot4(g, row4(a.v, j, kv, a.head_dim)) - delta) * a.scale, k);
        }
    }
    put4(a.d_q, t, h, a.head_dim, acc);
}

__global__ void attn_dkv_kernel(const __grid_constant__ PlainDev a) {
    const uint32_t kv = blockIdx.y, t = blockIdx.x * kWarps + threadIdx.x / 32;
    if (t >= a.n_tokens) return;
    const uint32_t group = a.q_heads / a.kv_heads;
    uint32_t first, end;
    float4 dk = make_float4(0.f, 0.f, 0.f, 0.f), dv = dk;
    if (sequence_of(a, t, &first, &end)) {
        const float4 k = row4(a.k, t, kv, a.head_dim), v = row4(a.v, t, kv, a.head_dim);
        for (uint32_t h = kv * group; h < (kv + 1) * group; ++h)
            for (uint32_t i = t; i < end; ++i) {
                const float4 q = row4(a.q, i, h, a.head_dim), g = row4(a.d_o, i, h, a.head_dim);
                const float p = expf(dot4(q, k) * a.scale - a.lse[size_t(h) * a.n_tokens + i]);
                add4(dv, p, g);
                add4(dk, p * (dot4(g, v) - a.delta[size_t(h) * a.n_tokens + i]) * a.scale, q);
            }
    }
    put4(a.d_k, t, kv, a.head_dim, dk);
    put4(a.d_v, t, kv, a.head_dim, dv);
}

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

struct Span {
    uint64_t lo, hi;
};
// Alignment, strides and extent of one [tokens][heads][dim] block; outputs need a place for every element.
int check_heads(const gac_attn_heads &h, const gac_attn &a, uint32_t heads, bool output, const char *name, Span *span) {
    const uint64_t p = reinterpret_cast<uint64_t>(h.p);
    if (!p || p % 16) return fail(nullptr, GAC_ERR_INVALID_ARG, "%s must be a 16-byte aligned device pointer", name);
    const int64_t most = int64_t(1) << 38;
    if (h.token < 0 || h.head < 0 || h.token > most || h.head > most || h.token % 8 || h.head % 8)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements, 0..2^38", name);
    const uint64_t nt = a.n_tokens, nh = heads, dim = a.head_dim;
    if (nt > 1 && h.token == 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "%s: tokens must not share one row", name);
    if (output) {
        const bool token_less = h.token <= h.head;
        const uint64_t less = token_less ? h.token : h.head, more = token_less ? h.head : h.token;
        const uint64_t n_less = token_less ? nt : nh, n_more = token_less ? nh : nt;
        if ((n_less > 1 && less < dim) || (n_more > 1 && more < (n_less - 1) * (n_less > 1 ? less : 0) + dim))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "%s: heads overlap one another", name);
    }
    span->lo = p;
    span->hi = p + ((nt - 1) * uint64_t(h.token) + (nh - 1) * uint64_t(h.head) + dim) * 2;
    return GAC_OK;
}

bool overlap(const Span &x, const Span &y) { return x.lo < y.hi && y.lo < x.hi; }

// Everything that does not look at pointers.
int check_shape(const gac_attn *args) {
    if (!args) return fail(nullptr, GAC_ERR_INVALID_ARG, "args is NULL%s");
    const gac_attn &a = *args;
    if (a.dtype != GAC_BF16) return fail(nullptr, GAC_ERR_DTYPE, "attention works on bfloat16%s");
    if (a.reserved != 0) return fail(nullptr, GAC_ERR_INVALID_ARG, "reserved field must be 0%s");
    if (a.head_dim < 8 || a.head_dim % 8 || a.head_dim > GAC_ATTN_MAX_HEAD_DIM)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "head_dim must be a multiple of 8, 8..%s%lld", "", GAC_ATTN_MAX_HEAD_DIM);
    if (a.kv_heads == 0 || a.q_heads == 0 || a.q_heads % a.kv_heads || a.q_heads > 4096)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads, 1..4096%s");
    if (a.n_tokens > (1u << 26) || a.n_seqs > (1u << 20))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "n_tokens <= 2^26 and n_seqs <= 2^20 are supported%s");
    if (!isfinite(a.scale)) return fail(nullptr, GAC_ERR_INVALID_ARG, "scale must be finite%s");
    return GAC_OK;
}

HeadsDev dev(const gac_attn_heads &h) { return HeadsDev{static_cast<char *>(h.p), 2 * h.token, 2 * h.head}; }

PlainDev dev_args(const gac_attn &a) {
    PlainDev d{};
    d.q = dev(a.q);
    d.k = dev(a.k);
    d.v = dev(a.v);
    d.o = dev(a.o);
    d.lse = a.lse;
    d.cu = a.cu_seqlens;
    d.n_tokens = a.n_tokens;
    d.n_seqs = a.n_seqs;
    d.q_heads = a.q_heads;
    d.kv_heads = a.kv_heads;
    d.head_dim = a.head_dim;
    d.scale = a.scale;
    return d;
}

// ------------------------------------------------------------ launches

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Describes one [tokens][heads][dim] operand for loads of kTile rows x 64 elements of one head.  Heads that
// share one memory (stride 0) are described as one head, and *mul makes the head coordinate 0.
int tensor_map(CUtensorMap *map, int *mul, const gac_attn_heads &h, const gac_attn &a, uint32_t heads) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail(nullptr, GAC_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled%s");
    const bool one = heads == 1 || h.head == 0;
    *mul = one ? 0 : 1;
    const uint64_t row = (uint64_t(a.head_dim) * 2 + 15) / 16 * 16;
    const cuuint64_t dims[3] = {a.head_dim, one ? 1u : heads, a.n_tokens};
    const cuuint64_t strides[2] = {one ? row : uint64_t(h.head) * 2, a.n_tokens == 1 ? row : uint64_t(h.token) * 2};
    const cuuint32_t box[3] = {64, 1, kTile}, steps[3] = {1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, h.p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(nullptr, GAC_ERR_CUDA, "cuTensorMapEncodeTiled refused an operand (CUresult %s%lld)", "", (long long)r);
    return GAC_OK;
}

RowsOut rows_out(const gac_attn_heads &h) { return RowsOut{static_cast<char *>(h.p), 2 * h.token, 2 * h.head}; }

AttnDev kernel_args(const gac_attn &a) {
    AttnDev d{};
    d.cu = a.cu_seqlens;
    d.n_tokens = a.n_tokens;
    d.n_seqs = a.n_seqs;
    d.q_heads = a.q_heads;
    d.kv_heads = a.kv_heads;
    d.head_dim = a.head_dim;
    d.scale = a.scale;
    d.exp2_scale = std::max(fabsf(a.scale) * kLog2e, 1e-37f);   // above zero, so that a hidden score stays -infinity
    d.negate = a.scale < 0.0f ? kNegateA : 0u;
    d.lse = a.lse;
    d.o = rows_out(a.o);
    return d;
}

// More dynamic shared memory than the default, asked for once per kernel and device.
template <typename K>
int allow_smem(K kernel, int bytes, int device, bool (&done)[64]) {
    if (device < 64 && done[device]) return GAC_OK;
    GAC_CUDA(nullptr, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (device < 64) done[device] = true;
    return GAC_OK;
}

int grid_of(uint32_t slots, uint32_t heads, uint32_t *grid) {
    const uint64_t n = uint64_t(slots) * heads;
    if (n > 0x7FFFFFFFull) return fail(nullptr, GAC_ERR_INVALID_ARG, "too many tokens, sequences and heads for one call%s");
    *grid = uint32_t(n);
    return GAC_OK;
}

template <int DP>
int launch_forward(const gac_attn &a, int device, cudaStream_t s) {
    static bool done[64];
    AttnDev d = kernel_args(a);
    CUtensorMap mq, mk, mv;
    if (int rc = tensor_map(&mq, &d.q_mul, a.q, a, a.q_heads)) return rc;
    if (int rc = tensor_map(&mk, &d.k_mul, a.k, a, a.kv_heads)) return rc;
    if (int rc = tensor_map(&mv, &d.v_mul, a.v, a, a.kv_heads)) return rc;
    uint32_t grid;
    if (int rc = grid_of(slot_count(a.n_tokens, a.n_seqs, 2 * kTile), a.q_heads, &grid)) return rc;
    if (int rc = allow_smem(attn_forward_kernel<DP>, Fwd<DP>::kSmem, device, done)) return rc;
    attn_forward_kernel<DP><<<grid, Fwd<DP>::kThreads, Fwd<DP>::kSmem, s>>>(mq, mk, mv, d);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

int check_pointers(const gac_attn &a, Span (&in)[3], Span *o) {
    if (int rc = check_heads(a.q, a, a.q_heads, false, "q", &in[0])) return rc;
    if (int rc = check_heads(a.k, a, a.kv_heads, false, "k", &in[1])) return rc;
    if (int rc = check_heads(a.v, a, a.kv_heads, false, "v", &in[2])) return rc;
    if (int rc = check_heads(a.o, a, a.q_heads, true, "o", o)) return rc;
    if (!a.lse || reinterpret_cast<uint64_t>(a.lse) % 4)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "lse must be a 4-byte aligned device pointer%s");
    if (!a.cu_seqlens || reinterpret_cast<uint64_t>(a.cu_seqlens) % 4)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "cu_seqlens must be a 4-byte aligned device pointer%s");
    for (const Span &s : in)
        if (overlap(s, *o)) return fail(nullptr, GAC_ERR_INVALID_ARG, "o overlaps an input%s");
    return GAC_OK;
}

}  // namespace

extern "C" {

size_t gac_attn_workspace(const gac_attn *args) {
    if (check_shape(args)) return 0;
    return std::max<size_t>(16, (size_t(args->q_heads) * args->n_tokens * 4 + 15) / 16 * 16);
}

int gac_attn_forward(const gac_attn *args, int cuda_device, void *cuda_stream) {
    if (int rc = check_shape(args)) return rc;
    const gac_attn &a = *args;
    if (a.n_tokens == 0) return GAC_OK;
    Span in[3], o;
    if (int rc = check_pointers(a, in, &o)) return rc;
    Range range("gac_attn_forward");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    return a.head_dim > 64 ? launch_forward<128>(a, cuda_device, static_cast<cudaStream_t>(cuda_stream))
                           : launch_forward<64>(a, cuda_device, static_cast<cudaStream_t>(cuda_stream));
}

int gac_attn_check(int cuda_device, void *cuda_stream) {
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int fault = 0;
    GAC_CUDA(nullptr, cudaMemcpyFromSymbolAsync(&fault, g_attn_fault, sizeof(fault), 0, cudaMemcpyDeviceToHost, s));
    GAC_CUDA(nullptr, cudaStreamSynchronize(s));
    if (!fault) return GAC_OK;
    const int none = 0;
    GAC_CUDA(nullptr, cudaMemcpyToSymbolAsync(g_attn_fault, &none, sizeof(none), 0, cudaMemcpyHostToDevice, s));
    GAC_CUDA(nullptr, cudaStreamSynchronize(s));
    return fail(nullptr, GAC_ERR_TIMEOUT, "a wait inside an attention kernel ran out%s");
}

int gac_attn_backward(const gac_attn *args, const gac_attn_grad *grad, int cuda_device, void *cuda_stream) {
    if (int rc = check_shape(args)) return rc;
    const gac_attn &a = *args;
    if (!grad) return fail(nullptr, GAC_ERR_INVALID_ARG, "grad is NULL%s");
    const gac_attn_grad &g = *grad;
    if (a.n_tokens == 0) return GAC_OK;
    Span in[5], out[3];
    {
        Span first[3];
        if (int rc = check_pointers(a, first, &in[3])) return rc;
        std::copy(first, first + 3, in);
    }
    if (int rc = check_heads(g.d_o, a, a.q_heads, false, "d_o", &in[4])) return rc;
    if (int rc = check_heads(g.d_q, a, a.q_heads, true, "d_q", &out[0])) return rc;
    if (int rc = check_heads(g.d_k, a, a.kv_heads, true, "d_k", &out[1])) return rc;
    if (int rc = check_heads(g.d_v, a, a.kv_heads, true, "d_v", &out[2])) return rc;
    for (const Span &x : in)
        for (const Span &y : out)
            if (overlap(x, y)) return fail(nullptr, GAC_ERR_INVALID_ARG, "a gradient overlaps an input%s");
    if (!g.workspace || reinterpret_cast<uint64_t>(g.workspace) % 16 || g.workspace_bytes < gac_attn_workspace(args))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "workspace must be 16-byte aligned and of gac_attn_workspace bytes%s");
    Range range("gac_attn_backward");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    PlainDev d = dev_args(a);
    d.d_o = dev(g.d_o);
    d.d_q = dev(g.d_q);
    d.d_k = dev(g.d_k);
    d.d_v = dev(g.d_v);
    d.delta = static_cast<float *>(g.workspace);
    const uint32_t nx = (a.n_tokens + kWarps - 1) / kWarps;
    attn_delta_kernel<<<dim3(nx, a.q_heads), kWarps * 32, 0, s>>>(d);
    attn_dq_kernel<<<dim3(nx, a.q_heads), kWarps * 32, 0, s>>>(d);
    attn_dkv_kernel<<<dim3(nx, a.kv_heads), kWarps * 32, 0, s>>>(d);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

}  // extern "C"
