"""Host-only checks of rotary positions with several axes and of the heads' norms: struct layouts, sections, argument
errors that are told before any device work, and the float64 forms the GPU tests compare with."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import build as gbuild

import heads_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    return gb.load_library()


def test_struct_layouts_match_the_header(tmp_path):
    names = ["gac_rotary_axes", "gac_norm", "gac_norm_grad"]
    fields = [(n, f) for n in names for f, _ in getattr(gb, n)._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gac.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", sizeof({n}));\n' for n in names)
                   + "".join(f'  printf("%zu\\n", offsetof({n}, {f}));\n' for n, f in fields) + "  return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    assert got == [ctypes.sizeof(getattr(gb, n)) for n in names] + [getattr(getattr(gb, n), f).offset for n, f in fields]
    for packed, struct in ((gb._AXES, gb.gac_rotary_axes), (gb._NORM, gb.gac_norm), (gb._NORM_GRAD, gb.gac_norm_grad)):
        assert packed.size == ctypes.sizeof(struct)


def test_sections():
    assert gb.gac_rotary_sections([2, 3, 1]).tolist() == [0, 0, 1, 1, 1, 2]
    assert gb.gac_rotary_sections([4, 2, 2], True).tolist() == [0, 1, 2, 0, 1, 2, 0, 0]
    assert gb.gac_rotary_sections([0, 2], True).tolist() == [1, 1]
    assert gb.gac_rotary_sections([3]).dtype == np.uint8


HEADS = gb.gac_rotary_heads * 2


def rotary_args(freqs, **over):
    a = gb.gac_rotary_args()
    a.qk[0] = gb.gac_rotary_heads(1 << 20, 1 << 24, 128, 64, 128, 64)
    a.heads[0], a.n_tokens, a.head_dim, a.rot_dim, a.scale = 2, 10, 64, 64, 1.0
    a.positions, a.freqs = 4096, ctypes.addressof(freqs)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def test_axes_errors_need_no_device(lib):
    freqs = (ctypes.c_double * 32)(*[1.0] * 32)
    good = (ctypes.c_uint8 * 32)(*[i % 3 for i in range(32)])
    bad = (ctypes.c_uint8 * 32)(*[3] * 32)

    def call(args=None, **over):
        on = gb.gac_rotary_axes(ctypes.addressof(good), 10, 3, 0)
        for k, v in over.items():
            setattr(on, k, v)
        a = rotary_args(freqs, **(args or {}))
        return lib.gac_rotary_on_axes(ctypes.byref(a), ctypes.byref(on), 0, None), lib.gac_last_error(None).decode()

    for over in ({"axis": None}, {"axis": ctypes.addressof(bad)}, {"stride": -1}, {"stride": 1 << 41}, {"n_axes": 0}, {"n_axes": 5},
                 {"n_axes": 2}, {"reserved": 1}, {"args": {"positions": None, "cu_seqlens": 4096}}, {"args": {"rot_dim": 0}},
                 {"args": {"positions": 4098}}, {"args": {"scale": math.nan}}):
        rc, msg = call(**over)
        assert rc == gb.GAC_ERR_INVALID_ARG and msg, over
    assert call(args={"n_tokens": 0})[0] == gb.GAC_OK
    assert lib.gac_rotary_on_axes(None, None, 0, None) == gb.GAC_ERR_INVALID_ARG


def test_norm_errors_need_no_device(lib):
    freqs = (ctypes.c_double * 32)(*[1.0] * 32)

    def forward(args=None, **over):
        a, n = rotary_args(freqs, **(args or {})), gb.gac_norm((ctypes.c_void_p * 2)(5 << 20, 6 << 20), 0, 0, 1e-6, 0.0)
        for k, v in over.items():
            setattr(n, k, v)
        return lib.gac_norm_rotary(ctypes.byref(a), None, ctypes.byref(n), 0, None), lib.gac_last_error(None).decode()

    two = (ctypes.c_void_p * 2)
    for over in ({"eps": 0.0}, {"eps": -1.0}, {"eps": math.inf}, {"eps": math.nan}, {"eps": 1e-50}, {"offset": math.nan}, {"reserved": 1},
                 {"weight": two((5 << 20) + 2, 0)}, {"weight": two(1 << 24, 0)}, {"weight": two(0, (1 << 24) + 2300)},
                 {"args": {"inverse": 1}}, {"args": {"rot_dim": 63}}, {"args": {"head_dim": 1032}}, {"args": {"positions": None}},
                 {"args": {"qk": HEADS(gb.gac_rotary_heads(1 << 20, (1 << 20) + 64, 128, 64, 128, 64))}}):
        rc, msg = forward(**over)
        assert rc == gb.GAC_ERR_INVALID_ARG and msg, over
    assert forward(weight_dtype=2)[0] == gb.GAC_ERR_DTYPE and forward(args={"dtype": 7})[0] == gb.GAC_ERR_DTYPE
    assert forward(args={"n_tokens": 0})[0] == gb.GAC_OK
    assert lib.gac_norm_rotary(None, None, None, 0, None) == gb.GAC_ERR_INVALID_ARG

    def heads(p, token=128, head=64):
        return gb.gac_attn_heads(p, token, head)

    def backward(args=None, norm=None, **over):
        a, n = rotary_args(freqs, **(args or {})), gb.gac_norm(two(5 << 20, 0), 0, 0, 1e-6, 0.0)
        g = gb.gac_norm_grad((gb.gac_attn_heads * 2)(heads(3 << 20), heads(0)), two(6 << 20, 0), 7 << 20, 1 << 20)
        for k, v in (norm or {}).items():
            setattr(n, k, v)
        for k, v in over.items():
            setattr(g, k, v)
        return lib.gac_norm_rotary_backward(ctypes.byref(a), None, ctypes.byref(n), ctypes.byref(g), 0, None), lib.gac_last_error(None).decode()

    one = lambda h: (gb.gac_attn_heads * 2)(h, heads(0))  # noqa: E731
    in_place = {"qk": HEADS(gb.gac_rotary_heads(1 << 20, 1 << 20, 128, 64, 128, 64))}
    for over in ({"workspace": None}, {"workspace": (7 << 20) + 4}, {"workspace_bytes": 10 * 2 * 64 * 4 - 1}, {"x": one(heads(0))},
                 {"x": one(heads((3 << 20) + 2))}, {"x": one(heads(3 << 20, -1))}, {"x": one(heads(1 << 24))},        # x and d_x
                 {"args": in_place, "x": one(heads(1 << 20))}, {"d_weight": two((6 << 20) + 2, 0)}, {"d_weight": two(6 << 20, (6 << 20) + 4)},
                 {"d_weight": two(5 << 20, 0)}, {"d_weight": two(3 << 20, 0)}, {"d_weight": two(1 << 20, 0)}, {"d_weight": two(1 << 24, 0)},
                 {"d_weight": two(7 << 20, 0)}, {"workspace": 1 << 20}, {"workspace": 1 << 24}, {"workspace": 3 << 20}, {"workspace": 5 << 20},
                 {"norm": {"eps": 0.0}}, {"args": {"inverse": 1}}):
        rc, msg = backward(**over)
        assert rc == gb.GAC_ERR_INVALID_ARG and msg, over
    assert lib.gac_norm_rotary_backward(None, None, None, None, 0, None) == gb.GAC_ERR_INVALID_ARG
    assert lib.gac_norm_rotary_workspace(None) == 0
    assert lib.gac_norm_rotary_workspace(ctypes.byref(rotary_args(freqs))) == 10 * 2 * 64 * 4
    assert lib.gac_norm_rotary_workspace(ctypes.byref(rotary_args(freqs, n_tokens=1 << 20))) == ref.SHARES * 2 * 64 * 4


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("axis", [None, [0, 1, 1, 0, 2, 2]])
def test_the_plain_gradient_is_the_derivative(layout, axis):
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(7, 3, 20, generator=gen, dtype=torch.float64, requires_grad=True), torch.randn(20, generator=gen, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(7, 3, 20, generator=gen, dtype=torch.float64)
    pos = torch.randint(0, 50, (7,) if axis is None else (3, 7), generator=gen).double()
    freqs = torch.tensor(1e2 ** (-np.arange(6) / 6))
    z = torch.view_as_complex(torch.zeros(7, 1, 6, 2, dtype=torch.float64))
    for i in range(6):
        p = pos if axis is None else pos[axis[i]]
        z[:, 0, i] = 1.5 * torch.exp(1j * p * freqs[i])
    n = x / (x.pow(2).mean(-1, keepdim=True) + 1e-3).sqrt() * (0.5 + w)
    a, b = ref.parts(12, layout)
    y = n.clone()
    turned = torch.complex(n[..., a].contiguous(), n[..., b].contiguous()) * z
    y[..., a], y[..., b] = turned.real, turned.imag
    want = torch.autograd.grad(y, (x, w), dy)
    cs = ref.wheel(pos, freqs, axis, 1.5)
    value, _ = ref.norm(x.detach(), w.detach(), cs, layout, 1.5, 1e-3, 0.5)
    assert float((value - y.detach()).abs().max()) < 1e-12
    (dx, _), (dw, _) = ref.norm_back(dy, x.detach(), w.detach(), cs, layout, 1.5, 1e-3, 0.5)
    assert float((dx - want[0]).abs().max()) < 1e-12 and float((dw - want[1]).abs().max()) < 1e-12
