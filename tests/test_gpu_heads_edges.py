"""Calls of the heads' norms, positions on axes and the divergence that are allowed and out of the way: key heads alone, many turns of
every group of lanes, the largest rows and lists, one buffer for many rows, calls that follow one another in one graph."""
import ctypes
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

import distill_ref
import heads_ref as ref
from packed_ref import within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dims", [(30011, 3, 1, 64, BF), (20003, 1, 5, 32, F), (9001, 1, 1, 256, BF), (9001, 7, 1, 20, BF), (70001, 1, 1, 8, F)], ids=str)
def test_every_group_of_lanes_takes_many_tokens(dims):
    tokens, qh, kh, dim, dtype = dims
    freqs = gb.gac_rotary_freqs(dim // 2, 1e4)
    q, k, w = randn((tokens, qh, dim), dtype, 1), randn((tokens, kh, dim), dtype, 2), randn((2, dim), F, 3)
    pos = torch.randint(0, 5000, (tokens,), device="cuda", dtype=torch.int32)
    cs = ref.wheel(pos.double(), torch.from_numpy(freqs).cuda())
    out = gb.gac_norm_rotary(q, k, w[0], w[1], freqs, positions=pos)
    dq, dk = randn(q.shape, dtype, 4), randn(k.shape, dtype, 5)
    back = gb.gac_norm_rotary_backward(dq, dk, q, k, w[0], w[1], freqs, positions=pos)
    for i, (x, d) in enumerate(((q, dq), (k, dk))):
        within(out[i], *ref.norm(x, w[i], cs, "half", 1.0, 1e-6, 0.0))
        dx, dw = ref.norm_back(d, x, w[i], cs, "half", 1.0, 1e-6, 0.0)
        within(back[i], *dx)
        within(back[2 + i], *dw)


@pytest.mark.parametrize("dim", [64, 30])
def test_key_heads_alone(dim):
    """The C call without query heads; the weight of the absent kind gets a sum over nothing."""
    lib, tokens = gb.load_library(), 37
    x, dy, w = randn((tokens, 2, dim), BF, 1), randn((tokens, 2, dim), BF, 2), randn((dim,), F, 3)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw = torch.full((2, dim), 7.0, device="cuda")
    freqs = gb.gac_rotary_freqs(dim // 2 // 2 * 2, 1e4)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    a = gb.gac_rotary_args()
    a.heads[1], a.n_tokens, a.head_dim, a.rot_dim, a.scale, a.dtype = 2, tokens, dim, 2 * freqs.size, 1.0, gb.GAC_BF16
    a.positions, a.freqs = pos.data_ptr(), freqs.ctypes.data
    a.qk[1] = gb.gac_rotary_heads(x.data_ptr(), y.data_ptr(), 2 * dim, dim, 2 * dim, dim)
    two = ctypes.c_void_p * 2
    norm = gb.gac_norm(two(0, w.data_ptr()), gb.GAC_F32, 0, 1e-6, 0.0)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.gac_norm_rotary(ctypes.byref(a), None, ctypes.byref(norm), 0, stream) == gb.GAC_OK
    cs = ref.wheel(pos.double(), torch.from_numpy(freqs).cuda())
    within(y, *ref.norm(x, w, cs, "half", 1.0, 1e-6, 0.0))
    a.qk[1] = gb.gac_rotary_heads(dy.data_ptr(), dx.data_ptr(), 2 * dim, dim, 2 * dim, dim)
    need = lib.gac_norm_rotary_workspace(ctypes.byref(a))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    heads = gb.gac_attn_heads * 2
    grad = gb.gac_norm_grad(heads(gb.gac_attn_heads(0, 0, 0), gb.gac_attn_heads(x.data_ptr(), 2 * dim, dim)), two(dw[0].data_ptr(), dw[1].data_ptr()),
                            work.data_ptr(), need)
    assert lib.gac_norm_rotary_backward(ctypes.byref(a), None, ctypes.byref(norm), ctypes.byref(grad), 0, stream) == gb.GAC_OK
    want, want_w = ref.norm_back(dy, x, w, cs, "half", 1.0, 1e-6, 0.0)
    within(dx, *want)
    within(dw[1], *want_w)
    assert bool((dw[0] == 0).all())
    # the gradient over the gradient that came in: the same bits
    keep, g = dx.clone(), dy.clone()
    a.qk[1] = gb.gac_rotary_heads(g.data_ptr(), g.data_ptr(), 2 * dim, dim, 2 * dim, dim)
    assert lib.gac_norm_rotary_backward(ctypes.byref(a), None, ctypes.byref(norm), ctypes.byref(grad), 0, stream) == gb.GAC_OK
    assert torch.equal(g, keep)


def test_nothing_behind_the_outputs_is_written():
    """Outputs between other values: strided views of one buffer, at odd places."""
    freqs = gb.gac_rotary_freqs(32, 1e4)
    for dtype, dim in ((BF, 64), (F, 64), (BF, 36), (F, 33)):
        big = randn((19, 9, dim), dtype, 1)
        keep = big.clone()
        x, w, pos = big[2:17, 3:7], randn((dim,), F, 2), torch.arange(15, dtype=torch.int32, device="cuda")
        want, _ = gb.gac_norm_rotary(x, None, w, None, freqs, positions=pos)
        gb.gac_norm_rotary(x, None, w, None, freqs, positions=pos, in_place=True)
        keep[2:17, 3:7] = want
        assert torch.equal(big, keep)


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["top", "reverse"])
def test_the_largest_rows_and_lists(dtype, kind):
    vocab = 1310720 // (2 if dtype == BF else 4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(3, vocab, generator=gen, device="cuda").to(dtype)
    ids = torch.randperm(vocab, generator=gen, device="cuda")[:1024].expand(3, 1024).to(torch.int32).contiguous()
    ids[1, 500:] = ids[1, :524].clone()
    ids[2, 0], ids[2, 1] = 0, vocab - 1
    x.scatter_(1, ids.long(), (3.0 + torch.randn(3, 1024, generator=gen, device="cuda")).to(dtype))
    values = torch.log_softmax(torch.randn(3, 1024, generator=gen, device="cuda"), 1) - 0.2
    want = distill_ref.distill(x, ids, values, kind, 1.0)
    within(gb.gac_distill(x, ids, values, kind), *want["loss"])
    loss, grad = gb.gac_distill(x, ids, values, kind, grad=True)
    within(loss, *want["loss"])
    within(grad, *want["grad"])
    more = torch.zeros(1, vocab + 8, dtype=dtype, device="cuda")
    for bad in ((more[:, :vocab + 1], ids[:1], values[:1]), (x, torch.zeros(3, 1025, dtype=torch.int32, device="cuda"), torch.zeros(3, 1025, device="cuda"))):
        with pytest.raises(gb.GacError) as e:
            gb.gac_distill(*bad)
        assert e.value.status == gb.GAC_ERR_INVALID_ARG


@pytest.mark.parametrize("size", [(60000, 40, 3), (3000, 2500, 20), (700, 33001, 9), (450, 151936, 5)], ids=str)
@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_many_rows_of_every_length(dtype, size):
    """Both shapes of the kernel, whole rows and split ones; some rows of each against the reference, and the calls against each other."""
    tokens, vocab, top = size
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(tokens, vocab, generator=gen, device="cuda").to(dtype)
    first = torch.randint(0, vocab, (tokens, 1), generator=gen, device="cuda")
    ids = ((first + torch.arange(top, device="cuda") * max(1, vocab // top)) % vocab).to(torch.int32)
    ids[::7] = -1
    values = torch.log_softmax(torch.randn(tokens, top, generator=gen, device="cuda"), 1) - 0.1
    w = torch.rand(tokens, generator=gen, device="cuda")
    loss, grad = gb.gac_distill(x, ids, values, "forward", weights=w, grad=True)
    alone = gb.gac_distill(x, ids, values, "forward")
    for part in (slice(0, 9), slice(tokens // 2, tokens // 2 + 9), slice(tokens - 9, tokens)):
        want = distill_ref.distill(x[part], ids[part], values[part], "forward", 1.0, w[part])
        within(loss[part], *want["loss"])
        within(alone[part], *want["loss"])
        within(grad[part], *want["grad"])
    # what every row's gradient adds up to: nothing, since the shares of all tokens add up to one
    total, size = grad.double().sum(1), grad.double().abs().sum(1)
    assert bool((total.abs() <= 2.0 ** (-8 if dtype == BF else -18) * size + 1e-30).all())
    assert bool((grad[::7] == 0).all()) and bool((loss[::7] == 0).all())


def test_one_teacher_for_all_rows():
    x, w = randn((50, 3001), F, 1), torch.rand(50, device="cuda")
    ids = torch.randperm(3001, device="cuda")[:8].to(torch.int32).expand(50, 8)          # stride 0
    values = torch.log_softmax(randn((8,), F, 2), 0).expand(50, 8) - 0.3 * 1.0
    values = values[:1].contiguous().expand(50, 8)
    loss, grad = gb.gac_distill(x, ids, values, "forward", weights=w, grad=True)
    want = distill_ref.distill(x, ids, values, "forward", 1.0, w)
    within(loss, *want["loss"])
    within(grad, *want["grad"])


def test_one_graph_for_a_whole_step():
    freqs, axis = gb.gac_rotary_freqs(64, 1e4), gb.gac_rotary_sections([8, 12, 12])
    q, k, w = randn((300, 4, 64), BF, 1), randn((300, 2, 64), BF, 2), randn((2, 64), F, 3)
    pos = torch.randint(0, 900, (3, 300), device="cuda", dtype=torch.int32)
    x, ids = randn((300, 1021), BF, 4), torch.randint(-1, 1021, (300, 12), device="cuda", dtype=torch.int32)
    values = torch.log_softmax(randn((300, 12), F, 5), 1) - 0.5

    def step():
        a = gb.gac_norm_rotary(q, k, w[0], w[1], freqs, positions=pos, axes=axis)
        b = gb.gac_norm_rotary_backward(*a, q, k, w[0], w[1], freqs, positions=pos, axes=axis)
        c = gb.gac_rotary(q, k, freqs, positions=pos, axes=axis, inverse=True)
        return [*a, *b, *c, *gb.gac_distill(x, ids, values, "reverse", grad=True)]

    want = step()
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(step())
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(math.isfinite(float(t.float().abs().max())) for t in want)
