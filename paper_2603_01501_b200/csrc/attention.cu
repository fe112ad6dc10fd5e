// Causal attention over a pack of sequences, grouped heads, forward and backward (gac_attn_* of include/gac.h): argument
// checks, operand descriptions and launches; the kernels and what bounds them are in attention_kernels.cuh.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <cstddef>
#include <type_traits>

#include "gac.h"
#include "gac_host.h"
#include "faults.h"
#include "overlap.h"
#include "attention_kernels.cuh"

namespace {

int fail(std::nullptr_t, int code, const char *fmt, const char *a = "", long long b = 0) {
    snprintf(g_init_err, sizeof(g_init_err), fmt, a, b);
    return code;
}

// Alignment, strides and extent of one [tokens][heads][dim] block; outputs need a place for every element.
int check_heads(const gac_attn_heads &h, const gac_attn &a, uint32_t heads, bool output, const char *name, Rows *rows) {
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
    *rows = Rows{p, uint64_t(h.token) * 2, uint64_t(h.head) * 2, nt, nh, dim * 2};
    return GAC_OK;
}

bool spans_cross(const Rows &x, const Rows &y) { return x.p < y.end() && y.p < x.end(); }
Rows block(const void *p, uint64_t bytes) { return Rows{reinterpret_cast<uint64_t>(p), 0, 0, 1, 1, bytes}; }
Rows lse_of(const gac_attn &a) { return block(a.lse, uint64_t(a.q_heads) * a.n_tokens * sizeof(float)); }

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
    if (uint64_t(a.n_tokens) * a.q_heads > (1ull << 31))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "n_tokens * q_heads <= 2^31 is supported%s");
    if (!isfinite(a.scale)) return fail(nullptr, GAC_ERR_INVALID_ARG, "scale must be finite%s");
    return GAC_OK;
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

// Limit of the waits inside a kernel, in units of 1024 ns.  The longest are for another warp to get through a job, one turn for
// each key (or query) tile of up to the whole pack and each of the job's heads: two seconds, and 20 us for each turn, which
// takes about 2 (backward, 28/4 heads x 128: 1.9).  At most 2^31 / 128 turns by check_shape.
uint32_t wait_limit(const gac_attn &a, uint32_t heads) { return uint32_t(2000000 + 20ull * (a.n_tokens / kTile + 1) * heads); }

AttnDev kernel_args(const gac_attn &a, uint32_t heads) {
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
    d.wait_limit = wait_limit(a, heads);
    d.lse = a.lse;
    d.o = rows_out(a.o);
    return d;
}

// Once per kernel and device: more dynamic shared memory than the default, and a look at the registers a CTA is
// launched with, where its warpgroups count on them.
template <typename K>
int allow_smem(K kernel, int bytes, int device, std::atomic<bool> (&done)[64], int regs = 0) {
    if (device < 64 && done[device]) return GAC_OK;
    cudaFuncAttributes attr;
    GAC_CUDA(nullptr, cudaFuncGetAttributes(&attr, kernel));
    if (attr.numRegs < regs) return fail(nullptr, GAC_ERR_CUDA, "a kernel was compiled to fewer registers than its warpgroups share out%s");
    GAC_CUDA(nullptr, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (device < 64) done[device] = true;
    return GAC_OK;
}

int grid_of(uint32_t count, uint32_t heads, uint32_t *grid) {
    const uint64_t n = uint64_t(count) * heads;
    if (n > 0x7FFFFFFFull) return fail(nullptr, GAC_ERR_INVALID_ARG, "too many tokens, sequences and heads for one call%s");
    *grid = uint32_t(n);
    return GAC_OK;
}

template <int DP>
int launch_forward(const gac_attn &a, int device, cudaStream_t s) {
    static std::atomic<bool> done[64];
    AttnDev d = kernel_args(a, 1);
    CUtensorMap mq, mk, mv;
    if (int rc = tensor_map(&mq, &d.q_mul, a.q, a, a.q_heads)) return rc;
    if (int rc = tensor_map(&mk, &d.k_mul, a.k, a, a.kv_heads)) return rc;
    if (int rc = tensor_map(&mv, &d.v_mul, a.v, a, a.kv_heads)) return rc;
    uint32_t grid;
    if (int rc = grid_of(job_count(a.n_tokens, a.n_seqs, 2 * kTile), a.q_heads, &grid)) return rc;
    if (int rc = allow_smem(attn_forward_kernel<DP>, Fwd<DP>::kSmem, device, done, Fwd<DP>::kRegs)) return rc;
    attn_forward_kernel<DP><<<grid, Fwd<DP>::kThreads, Fwd<DP>::kSmem, s>>>(mq, mk, mv, d);
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

// Query heads of a group are summed in one CTA as long as there are enough key tiles to go round; with fewer, parts
// of the group go to CTAs of their own and a second kernel adds them.  Backward with this limit, with 250 and with 600
// jobs: 8192 tokens, 12/2 heads 199 us, 225, 213; 16384 tokens in one sequence 2.33 ms, 2.90, 2.38; 12384 tokens, 28/4
// heads 0.99 ms, 1.00, 1.06.  Parts have equally many heads, so groups of prime size go from one part to one for each head.
constexpr uint32_t kEnoughJobs = 370;   // 2.5 per SM
uint32_t parts_of(const gac_attn &a) {
    const uint32_t group = a.q_heads / a.kv_heads;
    const uint64_t jobs = uint64_t(job_count(a.n_tokens, a.n_seqs, kTile)) * a.kv_heads;
    for (uint32_t parts = 1; parts < group; ++parts)
        if (group % parts == 0 && jobs * parts >= kEnoughJobs) return parts;
    return group;
}
size_t rows_bytes(const gac_attn &a) { return (size_t(a.q_heads) * a.n_tokens * sizeof(float2) + 15) / 16 * 16; }

template <typename... Args>
cudaError_t launch_next(void (*kernel)(Args...), uint32_t grid, uint32_t threads, uint32_t smem, cudaStream_t s, const std::remove_const_t<Args> &...args) {
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(grid);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = s;
    config.attrs = &early;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

template <int DP>
int launch_backward(const gac_attn &a, const gac_attn_grad &g, int device, cudaStream_t s) {
    static std::atomic<bool> done_kv[64], done_q[64];
    const uint32_t parts = parts_of(a);
    AttnDev d = kernel_args(a, a.q_heads / a.kv_heads / parts);
    d.d_q = rows_out(g.d_q);
    d.d_k = rows_out(g.d_k);
    d.d_v = rows_out(g.d_v);
    d.do_in = static_cast<const char *>(g.d_o.p);
    d.do_token = 2 * g.d_o.token;
    d.do_head = 2 * g.d_o.head;
    d.rows = static_cast<float2 *>(g.workspace);
    d.parts = parts;
    d.part_sums = reinterpret_cast<float *>(static_cast<char *>(g.workspace) + rows_bytes(a));
    CUtensorMap mq, mk, mv, mdo;
    if (int rc = tensor_map(&mq, &d.q_mul, a.q, a, a.q_heads)) return rc;
    if (int rc = tensor_map(&mk, &d.k_mul, a.k, a, a.kv_heads)) return rc;
    if (int rc = tensor_map(&mv, &d.v_mul, a.v, a, a.kv_heads)) return rc;
    if (int rc = tensor_map(&mdo, &d.do_mul, g.d_o, a, a.q_heads)) return rc;
    uint32_t grid_q, grid_kv;
    if (int rc = grid_of(job_count(a.n_tokens, a.n_seqs, 2 * kTile), a.q_heads, &grid_q)) return rc;
    if (int rc = grid_of(job_count(a.n_tokens, a.n_seqs, kTile), a.kv_heads * d.parts, &grid_kv)) return rc;
    if (int rc = allow_smem(attn_dq_kernel<DP>, BwdQ<DP>::kSmem, device, done_q, BwdQ<DP>::kRegs)) return rc;
    if (int rc = allow_smem(attn_dkv_kernel<DP>, BwdKv<DP>::kSmem, device, done_kv, BwdKv<DP>::kRegs)) return rc;
    const uint64_t units = uint64_t(a.q_heads) * a.n_tokens, per = kRowThreads / 16 * kRowsInFlight;
    attn_rows_kernel<<<uint32_t((units + per - 1) / per), kRowThreads, 0, s>>>(d);
    // each of the others is set up while the one before it ends, and waits for its results where it needs them
    GAC_CUDA(nullptr, launch_next(attn_dq_kernel<DP>, grid_q, BwdQ<DP>::kThreads, BwdQ<DP>::kSmem, s, mq, mk, mv, mdo, d));
    GAC_CUDA(nullptr, launch_next(attn_dkv_kernel<DP>, grid_kv, BwdKv<DP>::kThreads, BwdKv<DP>::kSmem, s, mq, mk, mv, mdo, d));
    if (d.parts > 1) {
        const uint64_t n = 2 * uint64_t(a.n_tokens) * a.kv_heads * (a.head_dim / 8);
        GAC_CUDA(nullptr, launch_next(attn_sum_parts_kernel, uint32_t((n + 255) / 256), 256, 0, s, d));
    }
    GAC_CUDA(nullptr, cudaGetLastError());
    return GAC_OK;
}

int check_pointers(const gac_attn &a, Rows (&in)[3], Rows *o) {
    if (int rc = check_heads(a.q, a, a.q_heads, false, "q", &in[0])) return rc;
    if (int rc = check_heads(a.k, a, a.kv_heads, false, "k", &in[1])) return rc;
    if (int rc = check_heads(a.v, a, a.kv_heads, false, "v", &in[2])) return rc;
    if (int rc = check_heads(a.o, a, a.q_heads, true, "o", o)) return rc;
    if (!a.lse || reinterpret_cast<uint64_t>(a.lse) % 4)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "lse must be a 4-byte aligned device pointer%s");
    if (!a.cu_seqlens || reinterpret_cast<uint64_t>(a.cu_seqlens) % 4)
        return fail(nullptr, GAC_ERR_INVALID_ARG, "cu_seqlens must be a 4-byte aligned device pointer%s");
    const Rows lse = lse_of(a);
    for (const Rows &r : in)
        if (spans_cross(r, *o) || share(r, lse)) return fail(nullptr, GAC_ERR_INVALID_ARG, "o or lse overlaps an input%s");
    if (share(*o, lse)) return fail(nullptr, GAC_ERR_INVALID_ARG, "lse overlaps o%s");
    return GAC_OK;
}

}  // namespace

extern "C" {

size_t gac_attn_workspace(const gac_attn *args) {
    if (check_shape(args)) return 0;
    const gac_attn &a = *args;
    const uint32_t parts = parts_of(a);
    const size_t sums = parts > 1 ? size_t(parts) * 2 * a.n_tokens * a.kv_heads * a.head_dim * sizeof(float) : 0;
    return std::max<size_t>(16, rows_bytes(a) + sums);
}

int gac_attn_forward(const gac_attn *args, int cuda_device, void *cuda_stream) {
    if (int rc = check_shape(args)) return rc;
    const gac_attn &a = *args;
    if (a.n_tokens == 0) return GAC_OK;
    Rows in[3], o;
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
    unsigned faults = 0;
    GAC_CUDA(nullptr, cudaMemcpyFromSymbolAsync(&faults, g_attn_faults, sizeof(faults), 0, cudaMemcpyDeviceToHost, s));
    GAC_CUDA(nullptr, cudaStreamSynchronize(s));
    static thread_local FaultLedger ledger;
    try {
        if (!ledger.news(cuda_device, cuda_stream, faults)) return GAC_OK;
    } catch (...) {   // out of memory: told again rather than not at all
        if (!faults) return GAC_OK;
    }
    return fail(nullptr, GAC_ERR_TIMEOUT, "a wait inside an attention kernel ran out%s");
}

int gac_attn_backward(const gac_attn *args, const gac_attn_grad *grad, int cuda_device, void *cuda_stream) {
    if (int rc = check_shape(args)) return rc;
    const gac_attn &a = *args;
    if (!grad) return fail(nullptr, GAC_ERR_INVALID_ARG, "grad is NULL%s");
    const gac_attn_grad &g = *grad;
    if (a.n_tokens == 0) return GAC_OK;
    Rows in[5], out[3];
    {
        Rows first[3];
        if (int rc = check_pointers(a, first, &in[3])) return rc;
        std::copy(first, first + 3, in);
    }
    if (int rc = check_heads(g.d_o, a, a.q_heads, false, "d_o", &in[4])) return rc;
    if (int rc = check_heads(g.d_q, a, a.q_heads, true, "d_q", &out[0])) return rc;
    if (int rc = check_heads(g.d_k, a, a.kv_heads, true, "d_k", &out[1])) return rc;
    if (int rc = check_heads(g.d_v, a, a.kv_heads, true, "d_v", &out[2])) return rc;
    if (!g.workspace || reinterpret_cast<uint64_t>(g.workspace) % 16 || g.workspace_bytes < gac_attn_workspace(args))
        return fail(nullptr, GAC_ERR_INVALID_ARG, "workspace must be 16-byte aligned and of gac_attn_workspace bytes%s");
    const Rows lse = lse_of(a), work = block(g.workspace, gac_attn_workspace(args));
    for (const Rows &x : in) {
        for (const Rows &y : out)
            if (spans_cross(x, y)) return fail(nullptr, GAC_ERR_INVALID_ARG, "a gradient overlaps an input%s");
        if (share(x, work)) return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace overlaps an input%s");
    }
    if (share(lse, work)) return fail(nullptr, GAC_ERR_INVALID_ARG, "the workspace overlaps lse%s");
    // spans of views of one fused gradient cross, their rows do not share memory
    for (int i = 0; i < 3; ++i)
        if (share(out[i], out[(i + 1) % 3]) || share(out[i], work) || share(out[i], lse))
            return fail(nullptr, GAC_ERR_INVALID_ARG, "two gradients, or a gradient and the workspace or lse, overlap%s");
    Range range("gac_attn_backward");
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return fail(nullptr, GAC_ERR_CUDA, "cudaSetDevice failed%s");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return a.head_dim > 64 ? launch_backward<128>(a, g, cuda_device, s) : launch_backward<64>(a, g, cuda_device, s);
}

}  // extern "C"
