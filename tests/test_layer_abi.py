"""Refusals of the operators around the recurrence, and their workspaces (host code only; nothing is launched)."""
import ctypes
import os

import pytest
import torch

from paper_2401_04658_amd import binding

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, VALUE = 1, 2, 3, 4, 5, 7
P = 0x10000   # an aligned "device pointer": a refusal comes before any use
BF16, F32 = binding.LA2_BF16, binding.LA2_F32
FWD, BWD = binding.LA2_OP_FWD, binding.LA2_OP_BWD


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.lib_path()):
        from paper_2401_04658_amd.build import build
        build()
    return binding.load()


def test_layer_norm(lib):
    def fwd(rows=4, width=64, dtype=BF16, stride=64, x=P, w=P, b=P, eps=1e-5, y=P, mean=P, rstd=P):
        return lib.la2_layer_norm_fwd(rows, width, dtype, stride, x, w, b, eps, y, mean, rstd, None)

    def bwd(rows=4, width=64, dtype=BF16, stride=64, x=P, dy=P, w=P, mean=P, rstd=P, dx=P, dw=P, db=P, ws=P, size=1 << 30):
        return lib.la2_layer_norm_bwd(rows, width, dtype, stride, x, dy, w, mean, rstd, dx, dw, db, ws, size, None)

    for call in (fwd, bwd):
        assert call(rows=-1) == SHAPE and call(width=-1) == SHAPE and call(rows=1 << 40, stride=1 << 20) == SHAPE
        assert call(dtype=3) == DTYPE and call(dtype=-1) == DTYPE
        assert call(stride=63) == ALIGN and call(x=P + 2) == ALIGN and call(rstd=P + 4) == ALIGN and call(w=P + 8) == ALIGN
        for name in ("x", "mean", "rstd"):
            assert call(**{name: None}) == NULL
        assert call(width=0) == 0
    assert fwd(y=None) == NULL and fwd(rows=0, x=None, y=None) == 0
    for eps in (-1.0, float("inf"), float("nan")):
        assert fwd(eps=eps) == VALUE
    assert bwd(dx=None) == NULL and bwd(dy=None) == NULL
    assert bwd(rows=0, dw=None, db=None) == 0
    need = lib.la2_layer_norm_workspace_bytes(100000, 2048, BF16)
    assert need > 0 and need % (2 * 2048 * 4) == 0
    big = dict(rows=100000, width=2048, stride=2048)
    assert bwd(**big, ws=None) == WORKSPACE and bwd(**big, size=need - 1) == WORKSPACE and bwd(**big, ws=P + 128) == WORKSPACE
    assert lib.la2_layer_norm_workspace_bytes(-1, 64, BF16) == 0 and lib.la2_layer_norm_workspace_bytes(4, 64, 9) == 0


def linear(lib, op, rows=64, k=64, n=64, dtype=BF16, act=0, sx=None, sw=None, sy=None, **given):
    desc = binding.la2_linear_desc(rows, k, n, dtype, act, k if sx is None else sx, k if sw is None else sw, n if sy is None else sy)
    names = ("x", "w", "bias", "residual", "y", "pre") if op == FWD else ("x", "w", "pre", "dy", "dx", "dw", "d_bias")
    at = dict.fromkeys(names, P)
    at.update(ws=P, size=1 << 40)
    at.update(given)
    fn = lib.la2_linear_fwd if op == FWD else lib.la2_linear_bwd
    return fn(ctypes.byref(desc), *[at[x] for x in names], at["ws"], at["size"], None)


def test_linear(lib):
    assert lib.la2_linear_fwd(None, *[P] * 7, 0, None) == NULL and lib.la2_linear_bwd(None, *[P] * 8, 0, None) == NULL
    for op in (FWD, BWD):
        assert linear(lib, op, rows=-1) == SHAPE and linear(lib, op, k=-1, sx=64, sw=64) == SHAPE and linear(lib, op, n=-1, sy=64) == SHAPE
        assert linear(lib, op, rows=1 << 40) == SHAPE
        assert linear(lib, op, sx=1 << 22) == SHAPE and linear(lib, op, dtype=F32, sw=1 << 21) == SHAPE
        assert linear(lib, op, dtype=3) == DTYPE
        assert linear(lib, op, act=4) == VALUE and linear(lib, op, act=-1) == VALUE
        assert linear(lib, op, sx=63) == ALIGN and linear(lib, op, sw=63) == ALIGN and linear(lib, op, sy=63) == ALIGN
        assert linear(lib, op, x=P + 2) == ALIGN and linear(lib, op, w=P + 8) == ALIGN and linear(lib, op, pre=P + 4) == ALIGN
    for name in ("x", "w", "y"):
        assert linear(lib, FWD, **{name: None}) == NULL
    assert linear(lib, BWD, dy=None) == NULL and linear(lib, BWD, act=1, pre=None) == NULL
    assert linear(lib, BWD, w=None) == NULL and linear(lib, BWD, x=None) == NULL
    assert linear(lib, BWD, dx=None, dw=None, d_bias=None) == 0   # nothing wanted
    assert linear(lib, FWD, rows=0, x=None, y=None) == 0 and linear(lib, FWD, n=0, y=None) == 0
    assert linear(lib, BWD, rows=0, dw=None, d_bias=None) == 0 and linear(lib, BWD, n=0, dx=None) == 0


def test_linear_workspace(lib):
    def need(op, rows, k, n, dtype=BF16, act=2, sx=None):
        return lib.la2_linear_workspace_bytes(ctypes.byref(binding.la2_linear_desc(rows, k, n, dtype, act, sx or k, k, n)), op)

    assert need(FWD, 8, 1001, 77) == 0                      # few rows read any row
    assert need(FWD, 8192, 2048, 2048) == 0                 # fills the device, whole pieces
    assert need(FWD, 8192, 2047, 2048) >= 2 * 2048 * (8192 + 2048)   # both operands are copied
    assert need(BWD, 8192, 2048, 2048) >= 2 * 8192 * 2048   # dz
    assert need(BWD, 8192, 2048, 2048, act=0) < 2 * 8192 * 2048
    assert need(BWD, 50, 64, 0) == 0 and need(BWD, 0, 64, 0) == 0 and need(BWD, 50, 0, 64) > 0 and need(FWD, 50, 0, 64) == 0
    assert need(FWD, -1, 8, 8) == 0 and need(FWD, 8, 8, 8, dtype=5) == 0 and need(9, 8192, 2047, 2048) == 0
    assert lib.la2_linear_workspace_bytes(None, FWD) == 0
    for op, rows, k, n in ((FWD, 100, 2047, 64), (BWD, 300, 128, 64)):
        size = need(op, rows, k, n)
        assert size > 0
        for bad in (dict(ws=None), dict(size=size - 1), dict(ws=P + 64)):
            assert linear(lib, op, rows=rows, k=k, n=n, act=2, **bad) == WORKSPACE


def test_beam_select(lib):
    def call(batch=2, beams=4, vocab=100, dtype=BF16, stride=100, logits=P, scores=P, finished=P, eos=2, out=P, parent=P, token=P, done=P,
             ws=P, size=1 << 40):
        return lib.la2_beam_select(batch, beams, vocab, dtype, stride, logits, scores, finished, eos, out, parent, token, done, ws, size, None)

    assert call(batch=-1) == SHAPE and call(beams=0) == SHAPE and call(beams=33) == SHAPE and call(vocab=0) == SHAPE
    assert call(vocab=(1 << 20) + 1, stride=1 << 21) == SHAPE and call(batch=16384) == SHAPE
    assert call(dtype=7) == DTYPE
    assert call(eos=100) == VALUE and call(eos=-2) == VALUE and call(eos=-1) == VALUE
    assert call(stride=99) == ALIGN and call(logits=P + 2) == ALIGN and call(parent=P + 4) == ALIGN
    for name in ("logits", "scores", "out", "parent", "token", "done"):
        assert call(**{name: None}) == NULL
    need = lib.la2_beam_select_workspace_bytes(2, 4, 100, BF16)
    assert need >= 8 * 4 * 8
    assert call(ws=None) == WORKSPACE and call(size=need - 1) == WORKSPACE and call(ws=P + 16) == WORKSPACE
    assert call(batch=0, logits=None) == 0
    assert lib.la2_beam_select_workspace_bytes(2, 33, 100, BF16) == 0


def test_beam_reorder(lib):
    def call(states=(P, P), n=None, batch=2, beams=4, row=64, parent=P):
        at = (ctypes.c_void_p * max(1, len(states)))(*states) if states is not None else None
        return lib.la2_beam_reorder(len(states) if n is None else n, at, batch, beams, row, parent, None)

    assert call(n=-1) == SHAPE and call(batch=-1) == SHAPE and call(beams=0) == SHAPE and call(beams=33) == SHAPE and call(row=-16) == SHAPE
    assert call(batch=65536) == SHAPE
    assert call(row=8) == ALIGN and call(states=(P, P + 8)) == ALIGN and call(parent=P + 4) == ALIGN
    assert call(parent=None) == NULL and call(states=(P, None)) == NULL and call(states=None, n=1) == NULL
    assert call(states=()) == 0 and call(batch=0) == 0 and call(row=0) == 0


def test_the_binding_refuses_what_is_no_tensor_or_does_not_fit(monkeypatch):
    monkeypatch.setattr(binding, "_on_gpu", lambda t, what: None)
    monkeypatch.setattr(binding, "_call", lambda entry, t, *args: entry(*args, 0))
    x, w, b = torch.zeros(8, 64).bfloat16(), torch.zeros(32, 64).bfloat16(), torch.zeros(32)
    y, v = torch.zeros(8, 32).bfloat16(), torch.zeros(8)
    for bad in (4096, True, "x"):
        for call in (lambda: binding.la2_layer_norm_fwd(x, weight=bad), lambda: binding.la2_layer_norm_fwd(x, out=bad),
                     lambda: binding.la2_layer_norm_bwd(x, x, bad, v), lambda: binding.la2_layer_norm_bwd(x, x, v, v, workspace=bad),
                     lambda: binding.la2_linear_fwd(x, bad), lambda: binding.la2_linear_fwd(x, w, bad),
                     lambda: binding.la2_linear_fwd(x, w, residual=bad), lambda: binding.la2_linear_fwd(x, w, workspace=bad),
                     lambda: binding.la2_linear_bwd(bad, x, w), lambda: binding.la2_linear_bwd(y, x, w, pre=bad),
                     lambda: binding.la2_beam_select(torch.zeros(2, 2, 9), bad), lambda: binding.la2_beam_select(bad, torch.zeros(2, 2)),
                     lambda: binding.la2_beam_reorder([bad], torch.zeros(2, 2, dtype=torch.int32))):
            with pytest.raises(TypeError):
                call()
    i32 = torch.zeros(2, 2, dtype=torch.int32)
    for call in (lambda: binding.la2_layer_norm_fwd(x, weight=b), lambda: binding.la2_layer_norm_fwd(x, weight=torch.ones(64).bfloat16()),
                 lambda: binding.la2_layer_norm_fwd(x.t()), lambda: binding.la2_layer_norm_fwd(x, out=x.float()),
                 lambda: binding.la2_layer_norm_fwd(x.view(2, 4, 64)[:, :3]), lambda: binding.la2_layer_norm_fwd(torch.zeros(())),
                 lambda: binding.la2_layer_norm_bwd(y, x, v, v), lambda: binding.la2_layer_norm_bwd(x, x, v[:7], v),
                 lambda: binding.la2_linear_fwd(x, w.t()), lambda: binding.la2_linear_fwd(x, w.float()), lambda: binding.la2_linear_fwd(x, w, b[:31]),
                 lambda: binding.la2_linear_fwd(x, w, residual=x), lambda: binding.la2_linear_fwd(x, w, act="tanh"),
                 lambda: binding.la2_linear_fwd(x, w, act=["relu"]), lambda: binding.la2_linear_fwd(x, w, out=y.float()),
                 lambda: binding.la2_linear_fwd(x, w, residual=y, out=torch.zeros(8, 40).bfloat16()[:, :32]),
                 lambda: binding.la2_linear_bwd(x, x, w), lambda: binding.la2_linear_bwd(y, x, w, pre=y[:7], act="relu"),
                 lambda: binding.la2_beam_select(torch.zeros(4, 9), b), lambda: binding.la2_beam_select(torch.zeros(2, 2, 9), torch.zeros(2, 3)),
                 lambda: binding.la2_beam_select(torch.zeros(2, 2, 9), torch.zeros(2, 2), torch.zeros(2, 2)),
                 lambda: binding.la2_beam_reorder([torch.zeros(3, 4)], i32), lambda: binding.la2_beam_reorder([torch.zeros(4, 4)], i32.long()),
                 lambda: binding.la2_beam_reorder([torch.zeros(4, 4), torch.zeros(4, 8)], i32),
                 lambda: binding.la2_beam_reorder([torch.zeros(4, 8)[:, :4]], i32)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        binding.la2_layer_norm_fwd(torch.zeros(8, 64, dtype=torch.float64))


def test_the_binding_wants_gpu_tensors_and_reports_statuses():
    x = torch.zeros(8, 64).bfloat16()
    for call in (lambda: binding.la2_layer_norm_fwd(x), lambda: binding.la2_layer_norm_bwd(x, x, x, x), lambda: binding.la2_linear_fwd(x, x),
                 lambda: binding.la2_linear_bwd(x, x, x), lambda: binding.la2_beam_select(x, x), lambda: binding.la2_beam_reorder([x], x)):
        with pytest.raises(ValueError):
            call()
    assert binding._module().beam_reorder([torch.zeros(66, 4)], torch.zeros(2, 33, dtype=torch.int32), 0) == SHAPE
    assert binding._module().layer_norm_fwd(x, None, None, -1.0, None, None, None, 0) == VALUE
