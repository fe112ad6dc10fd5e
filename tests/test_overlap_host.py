"""Which operands the calls refuse because they share memory: the rule against byte sets, and the refusals (no device work)."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2603_01501_b200 import binding as gb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_rule_against_byte_sets(tmp_path):
    rng = random.Random(3)

    def block():
        nt, nh, width = rng.choice([1, 1, 2, 3, 5]), rng.choice([1, 1, 2, 3]), rng.choice([2, 4, 8])
        return [rng.randrange(100, 160, 2), rng.choice([0, 6, 8, 12, 24, 24, 24, 48]), rng.choice([0, 2, 4, 8, 8, 16, 40]), nt, nh, width]

    def bytes_of(b):
        return {b[0] + i * b[1] + j * b[2] + x for i in range(b[3]) for j in range(b[4]) for x in range(b[5])}

    cases = [(block(), block()) for _ in range(4000)]
    src = tmp_path / "rule.cpp"
    src.write_text('#include <stdio.h>\n#include "overlap.h"\nint main() {\n    unsigned long long v[12];\n'
                   '    while (scanf("%llu %llu %llu %llu %llu %llu %llu %llu %llu %llu %llu %llu", v, v+1, v+2, v+3, v+4, v+5, v+6, v+7, v+8, '
                   'v+9, v+10, v+11) == 12)\n'
                   '        printf("%d\\n", share(Rows{v[0], v[1], v[2], v[3], v[4], v[5]}, Rows{v[6], v[7], v[8], v[9], v[10], v[11]}));\n}\n')
    exe = tmp_path / "rule"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2603_01501_b200", "csrc"), "-o", str(exe),
                    str(src)], check=True)
    told = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, a + b)) for a, b in cases), capture_output=True, text=True,
                          check=True).stdout.split()
    assert len(told) == len(cases)
    seen = [0, 0]
    for (a, b), got in zip(cases, told):
        really = bool(bytes_of(a) & bytes_of(b))
        exact = a[3] == 1 or b[3] == 1 or a[1] == 0 or b[1] == 0 or a[1] == b[1]
        assert (got == "1") == really if exact else (got == "1" or not really), (a, b)
        seen[really] += exact
    assert min(seen) > 300


def rotary(x0, y0, x1, y1, **over):
    """gac_rotary on 10 tokens x 2 and 10 x 1 heads of 64 float32 elements, tokens 1024 bytes apart unless said."""
    freqs = (ctypes.c_double * 32)(*[1.0] * 32)
    a = gb.gac_rotary_args()
    token = over.get("token", 256)
    a.qk[0] = gb.gac_rotary_heads(x0, y0, token, 64, token, 64)
    a.qk[1] = gb.gac_rotary_heads(x1, y1, token, 64, token, 64)
    a.heads[0], a.heads[1], a.n_tokens, a.head_dim, a.rot_dim, a.scale = 2, 1, 10, 64, 64, 1.0
    a.positions, a.freqs = 4096, ctypes.addressof(freqs)
    return gb.load_library().gac_rotary(ctypes.byref(a), 0, None), gb.load_library().gac_last_error(None).decode()


M = 1 << 20


@pytest.mark.parametrize("x0,y0,x1,y1", [
    (M, M, M, M),                        # q and k in place on the same memory
    (M, M, M + 256, M + 256),            # k in place on q's second head
    (M, M, 2 * M, M),                    # q in place, k written over it
    (M, M, 2 * M, M + 1024),             # the same, one token later
    (2 * M, M, M, M),                    # k in place, q written over it
    (M, 3 * M, 2 * M, 3 * M),            # one output for both
    (M, 3 * M, 2 * M, 3 * M + 128),      # a part of it
    (M, 2 * M, 2 * M, 3 * M),            # q written where k is read
], ids=str)
def test_rotary_operands_that_share_memory_are_refused(x0, y0, x1, y1):
    rc, msg = rotary(x0, y0, x1, y1)
    assert rc == gb.GAC_ERR_INVALID_ARG and "overlap" in msg


def attention(backward=False, **over):
    """Forward or backward on 100 tokens, 4/2 heads x 64; the operands a megabyte apart unless said."""
    names = ("q", "k", "v", "o", "d_o", "d_q", "d_k", "d_v")
    at = {n: (i + 1) << 20 for i, n in enumerate(names)}
    at.update(lse=20 << 20, cu=21 << 20, workspace=22 << 20)
    at.update(over)
    h = {n: gb.gac_attn_heads(at[n], 256, 64) for n in names}
    a = gb.gac_attn(h["q"], h["k"], h["v"], h["o"], at["lse"], at["cu"], 100, 3, 4, 2, 64, gb.GAC_BF16, 0.125, 0)
    L = gb.load_library()
    if backward:
        g = gb.gac_attn_grad(h["d_o"], h["d_q"], h["d_k"], h["d_v"], at["workspace"], 1 << 20)
        rc = L.gac_attn_backward(ctypes.byref(a), ctypes.byref(g), 0, None)
    else:
        rc = L.gac_attn_forward(ctypes.byref(a), 0, None)
    return rc, L.gac_last_error(None).decode()


@pytest.mark.parametrize("over", [{"lse": M}, {"lse": 4 * M}, {"lse": 4 * M + 50_000}, {"lse": 2 * M - 4}], ids=str)
def test_attention_statistics_on_an_operand_are_refused(over):
    rc, msg = attention(**over)
    assert rc == gb.GAC_ERR_INVALID_ARG and "overlap" in msg


@pytest.mark.parametrize("over", [{"d_k": 6 * M + 128}, {"d_v": 7 * M + 512}, {"d_v": 6 * M + 16}, {"workspace": M + 16}, {"workspace": 5 * M - 64},
                                  {"workspace": 20 * M}, {"workspace": 6 * M + 64}, {"lse": 8 * M + 4}], ids=str)
def test_gradients_and_workspace_that_share_memory_are_refused(over):
    rc, msg = attention(backward=True, **over)
    assert rc == gb.GAC_ERR_INVALID_ARG and ("overlap" in msg or "same memory" in msg)
