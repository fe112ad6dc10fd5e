"""Host-only checks of the operators on packed rollouts: struct layouts, frequencies, argument errors that
are told before any device work, and the float64 forms the GPU tests compare with."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import build as gbuild

import packed_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    return gb.load_library()


def test_struct_layouts_match_the_header(tmp_path):
    names = ["gac_clip_tensor", "gac_clip_result", "gac_rotary_heads", "gac_rotary_args", "gac_attn_heads", "gac_attn",
             "gac_attn_grad"]
    fields = [(n, f) for n in names for f, _ in getattr(gb, n)._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gac.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", sizeof({n}));\n' for n in names)
                   + "".join(f'  printf("%zu\\n", offsetof({n}, {f}));\n' for n, f in fields) + "  return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    want = [ctypes.sizeof(getattr(gb, n)) for n in names] + [getattr(getattr(gb, n), f).offset for n, f in fields]
    assert got == want
    # the packed forms the calls send have the same layout
    for packed, struct in ((gb._ROTARY, gb.gac_rotary_args), (gb._ATTN, gb.gac_attn), (gb._ATTN_GRAD, gb.gac_attn_grad)):
        assert packed.size == ctypes.sizeof(struct)


def test_rotary_frequencies(lib):
    f = gb.gac_rotary_freqs(64, 1e4)
    assert np.allclose(f, 1e4 ** (-np.arange(0, 64, 2) / 64), rtol=1e-14, atol=0)
    assert np.allclose(gb.gac_rotary_freqs(64, 1e4, "linear", 8.0), f / 8, rtol=1e-14, atol=0)
    b = gb.gac_rotary_freqs(64, 1e4, "base", 8.0)
    assert b[0] == 1.0 and abs(b[-1] / f[-1] - 1 / 8) < 1e-12 and bool((np.diff(np.log(b / f)) < 0).all())
    p = gb.gac_rotary_freqs(64, 1e4, "parts", 8.0, trained=1024.0, low=1.0, high=4.0)
    turns = 1024.0 * f / (2 * math.pi)
    assert np.array_equal(p[turns >= 4.0], f[turns >= 4.0])
    assert np.allclose(p[turns <= 1.0], f[turns <= 1.0] / 8, rtol=1e-14, atol=0)
    mid = (turns > 1.0) & (turns < 4.0)
    assert mid.any() and bool(((p < f) & (p > f / 8))[mid].all())
    for bad in ((63, 1e4), (0, 1e4), (512, 1e4), (64, 1.0), (64, math.inf)):
        with pytest.raises(gb.GacError):
            gb.gac_rotary_freqs(*bad)
    for kw in ({"factor": 2.0}, {"scaling": "linear", "factor": 0.5}, {"scaling": "parts", "factor": 2.0, "trained": 0.0},
               {"scaling": "parts", "factor": 2.0, "low": 4.0, "high": 4.0}):
        with pytest.raises(gb.GacError):
            gb.gac_rotary_freqs(64, 1e4, **kw)
    with pytest.raises(gb.GacError):
        gb.gac_rotary_freqs(2, 1e4, "base", 2.0)


def test_argument_errors_need_no_device(lib):
    clip = (gb.gac_clip_tensor * 1)
    out = ctypes.c_void_p()

    def init(*entry):
        return lib.gac_clip_init(ctypes.byref(out), clip(gb.gac_clip_tensor(*entry)), 1, 0)

    assert init(0, 4096, 5, 0, 0) == gb.GAC_ERR_INVALID_ARG
    assert init(4096, 8192, 5, 2, 0) == gb.GAC_ERR_DTYPE
    assert init(4096, 8192, 5, 0, 1) == gb.GAC_ERR_INVALID_ARG
    assert init(4098, 8192, 5, 0, 0) == gb.GAC_ERR_INVALID_ARG
    assert init(4096, 4100, 5, 0, 0) == gb.GAC_ERR_INVALID_ARG
    assert lib.gac_clip_init(None, clip(), 1, 0) == gb.GAC_ERR_INVALID_ARG

    freqs = (ctypes.c_double * 32)(*[1.0] * 32)

    def rotary(**over):
        a = gb.gac_rotary_args()
        a.qk[0] = gb.gac_rotary_heads(1 << 20, 1 << 24, 128, 64, 128, 64)
        a.heads[0], a.n_tokens, a.head_dim, a.rot_dim, a.scale = 2, 10, 64, 64, 1.0
        a.positions, a.freqs = 4096, ctypes.addressof(freqs)
        for k, v in over.items():
            setattr(a, k, v)
        return lib.gac_rotary(ctypes.byref(a), 0, None), lib.gac_last_error(None).decode()

    for over in ({"rot_dim": 63}, {"rot_dim": 66}, {"rot_dim": 0}, {"layout": 2}, {"inverse": 2}, {"reserved": 1}, {"freqs": None},
                 {"scale": math.nan}, {"positions": None}, {"positions": 4098}, {"head_dim": 2000},
                 {"qk": (gb.gac_rotary_heads * 2)(gb.gac_rotary_heads(1 << 20, (1 << 20) + 64, 128, 64, 128, 64))},   # overlap
                 {"qk": (gb.gac_rotary_heads * 2)(gb.gac_rotary_heads(1 << 20, 1 << 24, 128, 64, 128, 32))},          # heads on heads
                 {"qk": (gb.gac_rotary_heads * 2)(gb.gac_rotary_heads(1 << 20, 1 << 20, 128, 64, 256, 64))},          # strides differ
                 {"qk": (gb.gac_rotary_heads * 2)(gb.gac_rotary_heads(1 << 20, 1 << 24, -128, 64, 128, 64))}):
        rc, msg = rotary(**over)
        assert rc == gb.GAC_ERR_INVALID_ARG and msg, over
    assert rotary(dtype=5)[0] == gb.GAC_ERR_DTYPE
    assert rotary(n_tokens=0)[0] == gb.GAC_OK

    def heads(p, token=256, head=64):
        return gb.gac_attn_heads(p, token, head)

    def attn(grad=None, **over):
        a = gb.gac_attn(heads(1 << 20), heads(2 << 20), heads(3 << 20), heads(4 << 20), 5 << 20, 6 << 20, 100, 3, 4, 2, 64, 1, 0.125, 0)
        for k, v in over.items():
            setattr(a, k, v)
        if grad is None:
            return lib.gac_attn_forward(ctypes.byref(a), 0, None)
        g = gb.gac_attn_grad(heads(7 << 20), heads(8 << 20), heads(9 << 20), heads(10 << 20), 11 << 20, 1 << 20)
        for k, v in grad.items():
            setattr(g, k, v)
        return lib.gac_attn_backward(ctypes.byref(a), ctypes.byref(g), 0, None)

    for over in ({"head_dim": 60}, {"head_dim": 136}, {"head_dim": 0}, {"q_heads": 3}, {"kv_heads": 0}, {"scale": math.inf},
                 {"reserved": 1}, {"lse": None}, {"cu_seqlens": 6 * 1024 + 2}, {"q": heads((1 << 20) + 8)}, {"k": heads(2 << 20, 256, 60)},
                 {"v": heads(3 << 20, -256)}, {"o": heads(4 << 20, 256, 56)}, {"o": heads(1 << 20)}, {"n_tokens": 1 << 27}):
        assert attn(**over) == gb.GAC_ERR_INVALID_ARG, over
        assert lib.gac_last_error(None).decode()
    assert attn(dtype=0) == gb.GAC_ERR_DTYPE
    assert attn(n_tokens=0) == gb.GAC_OK
    for over in ({"workspace": None}, {"workspace": (11 << 20) + 4}, {"workspace_bytes": 100}, {"d_q": heads(1 << 20)},
                 {"d_k": heads(4 << 20)}, {"d_v": heads(7 << 20)}, {"d_v": heads(9 << 20)}, {"workspace": 8 << 20}):
        assert attn(grad=over) == gb.GAC_ERR_INVALID_ARG, over
    assert lib.gac_attn_forward(None, 0, None) == gb.GAC_ERR_INVALID_ARG
    assert lib.gac_attn_backward(None, None, 0, None) == gb.GAC_ERR_INVALID_ARG
    assert lib.gac_attn_workspace(None) == 0


def test_the_plain_gradient_is_the_derivative():
    """The float64 form the kernels are compared with, against autograd of a dense softmax."""
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(13, n, 8, generator=gen, dtype=torch.float64, requires_grad=True) for n in (4, 2, 2))
    d_o = torch.randn(13, 4, 8, generator=gen, dtype=torch.float64)
    cu = [0, 4, 4, 12]
    seq = torch.tensor([0] * 4 + [2] * 8 + [9])
    seen = (seq[:, None] == seq[None]) & (torch.arange(13)[None] <= torch.arange(13)[:, None]) & (seq[:, None] < 9)
    S = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(2, 1)) * 0.3
    P = torch.where(seen, torch.exp(S), 0.0)
    P = P / P.sum(-1, keepdim=True).clamp(min=1e-300)
    o = torch.einsum("hij,jhd->ihd", P, v.repeat_interleave(2, 1))
    want = [o] + list(torch.autograd.grad(o, (q, k, v), d_o))
    got = packed_ref.attention(q.detach(), k.detach(), v.detach(), cu, 0.3, d_o)
    for name, w in zip(("o", "dq", "dk", "dv"), want):
        assert float((got[name][0] - w.detach()).abs().max()) < 1e-12
