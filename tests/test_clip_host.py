"""What the clipping calls of the binding refuse before the library is asked, and what the clipper keeps (no GPU)."""
import types

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed


class Fake:
    """What the checks look at of a tensor on some device."""

    def __init__(self, device, dtype):
        self.device, self.dtype, self.is_cuda = torch.device(device), dtype, True

    def numel(self):
        return 1

    def data_ptr(self):
        return 4096


class Library:
    def __getattr__(self, name):
        def call(*_):
            raise AssertionError(f"{name} was called")
        return call


def test_results_on_another_device_than_the_list_are_refused(monkeypatch):
    monkeypatch.setattr(gb, "load_library", Library)
    monkeypatch.setattr(gb, "_on", lambda stream, device: (0, None))
    ctx = types.SimpleNamespace(handle=None, device=torch.device("cuda", 0))
    here, there = Fake("cuda:0", torch.float64), Fake("cuda:1", torch.float64)
    norm = Fake("cuda:1", torch.float32)
    for call in (lambda: gb.gac_clip_grad_norm(ctx, 1.0, norm_out=norm), lambda: gb.gac_clip_sumsq(ctx, there),
                 lambda: gb.gac_clip_apply(ctx, there, 1.0), lambda: gb.gac_clip_apply(ctx, here, 1.0, norm_out=norm)):
        with pytest.raises(ValueError):
            call()


@pytest.fixture
def library(monkeypatch):
    """Stand-ins for the rule in exchange mode (a safe step, g unchanged) and for clipping; `calls` records the latter."""
    calls = types.SimpleNamespace(made=[], clipped=0, result=dict(g_set=0, out_set=0), next=0)

    def stats(ctx, t, staleness=0):
        return types.SimpleNamespace(regime=gb.GAC_REGIME_SAFE, nonfinite=0, **calls.result)

    def make(grads, *_, **__):
        calls.made.append([g.data_ptr() for g in grads])
        return types.SimpleNamespace(handle=len(calls.made))

    def clip(ctx, max_norm, eps=1e-6, norm_out=None, stream=None, fetch=False):
        calls.clipped += 1

    def project(ctx):
        calls.next ^= 1

    for name, f in (("gac_init", lambda g, d, hp: object()), ("gac_stats", stats), ("gac_project", project),
                    ("gac_next_gradient_set", lambda ctx: calls.next), ("gac_free", lambda ctx: None),
                    ("gac_clip_init", make), ("gac_clip_rebind", lambda *_, **__: None), ("gac_clip_grad_norm", clip), ("gac_clip_free", lambda ctx: None)):
        monkeypatch.setattr(gb, name, f, raising=False)
    return calls


def test_the_stored_direction_of_an_exchange_step_is_not_clipped(library):
    from paper_2603_01501_b200.controller import GradientAlignmentController
    params = [torch.nn.Parameter(torch.zeros(n)) for n in (3, 5)]
    controller, clipper = GradientAlignmentController(params, exchange=True), packed.GradientClipper(params)
    for p in params:
        p.grad = torch.ones_like(p)
    controller.step()                       # safe: .grad is the stored direction itself
    with pytest.raises(RuntimeError, match="clip_max_norm"):
        clipper.clip(1.0)
    assert library.clipped == 0
    controller.zero_grad()                  # the free tensors
    clipper.clip(1.0)
    library.result = dict(g_set=1, out_set=0)
    controller.step()                       # a projection: written into the free tensors, which may be clipped
    clipper.clip(1.0)
    assert library.clipped == 2


def test_the_clipper_rebinds_moved_gradients_and_survives_a_failure(library, monkeypatch):
    moved, kept = [], {}
    monkeypatch.setattr(gb, "gac_clip_rebind", lambda ctx, grads, *_, **__: moved.append([g.data_ptr() for g in grads]), raising=False)
    make = gb.gac_clip_init
    monkeypatch.setattr(gb, "gac_clip_init", lambda grads, *a, **kw: (kept.update(kw), make(grads))[1])
    params = [torch.nn.Parameter(torch.zeros(n)) for n in (3, 5)]
    clipper = packed.GradientClipper(params)

    def new_gradients():
        old = [p.grad for p in params]                  # alive, so that the new ones lie elsewhere
        for p in params:
            p.grad = torch.ones_like(p)
        return old

    new_gradients()
    clipper.clip(1.0)
    clipper.clip(1.0)
    assert len(library.made) == 1 and moved == [] and kept == {"keep": False}
    old = new_gradients()
    clipper.clip(1.0)
    assert len(library.made) == 1 and moved == [[p.grad.data_ptr() for p in params]]
    params[1].grad = None                               # another list
    clipper.clip(1.0)
    assert len(library.made) == 2 and len(moved) == 1

    def broken(*_, **__):
        raise gb.GacError(gb.GAC_ERR_CUDA, "no")
    good = gb.gac_clip_rebind, gb.gac_clip_init
    monkeypatch.setattr(gb, "gac_clip_rebind", broken)
    monkeypatch.setattr(gb, "gac_clip_init", broken)
    params[0].grad = torch.ones_like(params[0])
    for _ in range(2):                                  # fails, and does not take the old table for the new one
        with pytest.raises(gb.GacError):
            clipper.clip(1.0)
    params[1].grad = torch.ones_like(params[1])
    for _ in range(2):
        with pytest.raises(gb.GacError):
            clipper.clip(1.0)
    before = library.clipped
    monkeypatch.setattr(gb, "gac_clip_rebind", good[0])
    monkeypatch.setattr(gb, "gac_clip_init", good[1])
    clipper.clip(1.0)
    assert len(library.made) == 3 and library.clipped == before + 1 and len(old) == 2


def test_a_norm_that_is_not_finite_is_raised_when_asked_for(library, monkeypatch):
    def clip(ctx, max_norm, eps=1e-6, norm_out=None, stream=None, fetch=False):
        library.clipped += 1
        return types.SimpleNamespace(nonfinite=1, norm=float("nan"), timed_out=0) if fetch else None
    monkeypatch.setattr(gb, "gac_clip_grad_norm", clip)
    p = torch.nn.Parameter(torch.zeros(3))
    p.grad = torch.ones(3)
    clipper = packed.GradientClipper([p])
    clipper.clip(1.0)                                    # as it is, without waiting for the host
    with pytest.raises(gb.GacError) as e:
        clipper.clip(1.0, error_if_nonfinite=True)
    assert e.value.status == gb.GAC_ERR_NONFINITE and library.clipped == 2


def test_the_norm_is_float32_whatever_the_default_is():
    before = torch.get_default_dtype()
    try:
        torch.set_default_dtype(torch.bfloat16)
        assert packed.GradientClipper([torch.nn.Parameter(torch.zeros(3))]).norm.dtype is torch.float32
    finally:
        torch.set_default_dtype(before)
