"""Host-only checks of the divergence from a teacher's top logits: struct layout, argument errors that are told before any
device work, and the float64 form the GPU tests compare with."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import build as gbuild

import distill_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    return gb.load_library()


def test_struct_layout_matches_the_header(tmp_path):
    fields = [f for f, _ in gb.gac_distill_args._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gac.h"\nint main(void) {\n  printf("%zu\\n", sizeof(gac_distill_args));\n'
                   + "".join(f'  printf("%zu\\n", offsetof(gac_distill_args, {f}));\n' for f in fields) + "  return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    assert got == [ctypes.sizeof(gb.gac_distill_args)] + [getattr(gb.gac_distill_args, f).offset for f in fields]
    assert gb._DISTILL.size == ctypes.sizeof(gb.gac_distill_args)


def test_argument_errors_need_no_device(lib):
    def call(**over):
        a = gb.gac_distill_args(1 << 20, 1000, 2 << 20, 16, 3 << 20, 16, 4 << 20, 5 << 20, 6 << 20, 1000, 20, 1000, 16, 0, 0, 0, 1.0, 0)
        for k, v in over.items():
            setattr(a, k, v)
        return lib.gac_distill(ctypes.byref(a), 0, None), lib.gac_last_error(None).decode()

    for over in ({"kind": 3}, {"kind": -1}, {"reserved": 1}, {"temperature": 0.0}, {"temperature": -1.0}, {"temperature": math.nan},
                 {"temperature": math.inf}, {"temperature": 1e-4}, {"vocab": 0}, {"vocab": (1 << 20) + 1}, {"top": 0}, {"top": 1025},
                 {"n_tokens": (1 << 27) + 1}, {"loss": None, "d_logits": None}, {"logits": None}, {"ids": None}, {"teacher": None},
                 {"logits": (1 << 20) + 2}, {"ids": (2 << 20) + 2}, {"teacher": (3 << 20) + 1}, {"weights": (4 << 20) + 2},
                 {"loss": (5 << 20) + 2}, {"d_logits": (6 << 20) + 1}, {"logits_row": -1}, {"ids_row": 1 << 41}, {"teacher_row": -5},
                 {"d_row": 999}, {"loss": 6 << 20}, {"loss": 1 << 20}, {"loss": 2 << 20}, {"loss": 3 << 20}, {"loss": 4 << 20},
                 {"d_logits": (1 << 20) + 4}, {"d_logits": 1 << 20, "d_row": 1001}, {"d_logits": 2 << 20}, {"d_logits": 3 << 20},
                 {"d_logits": 4 << 20}, {"d_logits": 1 << 20, "loss": 1 << 20}):
        rc, msg = call(**over)
        assert rc == gb.GAC_ERR_INVALID_ARG and msg, over
    assert call(dtype=2)[0] == gb.GAC_ERR_DTYPE and call(teacher_dtype=-1)[0] == gb.GAC_ERR_DTYPE
    assert call(n_tokens=0)[0] == gb.GAC_OK
    assert lib.gac_distill(None, 0, None) == gb.GAC_ERR_INVALID_ARG


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_the_plain_gradient_is_the_derivative(kind):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(4, 50, generator=gen, dtype=torch.float64)
    ids = torch.stack([torch.randperm(50, generator=gen)[:6] for _ in range(4)]).to(torch.int32)
    teacher = torch.randn(4, 6, generator=gen, dtype=torch.float64).log_softmax(1) - 0.1
    leaf = x.clone().requires_grad_()
    lq = torch.log_softmax(leaf / 1.3, 1)
    at = lq.gather(1, ids.long())
    if kind == "top":
        lp = torch.log_softmax(teacher / 1.3, 1)
        loss = (lp.exp() * (lp - at)).sum(1)
    else:
        rest_p, rest_q = torch.log1p(-teacher.exp().sum(1)), torch.log1p(-at.exp().sum(1))
        if kind == "forward":
            loss = (teacher.exp() * (teacher - at)).sum(1) + rest_p.exp() * (rest_p - rest_q)
        else:
            loss = (at.exp() * (at - teacher)).sum(1) + rest_q.exp() * (rest_q - rest_p)
    w = torch.tensor([1.0, 2.0, 0.5, 0.0], dtype=torch.float64)
    want, = torch.autograd.grad((loss * w).sum(), leaf)
    got = ref.distill(x, ids, teacher, kind, 1.3, w)
    assert float((got["loss"][0] - loss.detach()).abs().max()) < 1e-12
    assert float((got["grad"][0] - want).abs().max()) < 1e-12
