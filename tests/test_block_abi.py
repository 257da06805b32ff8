"""Host-side checks of the operators in gdn_block.h: exported symbols, workspace sizes and refused arguments (no kernel
is launched: addresses are made up, or the tensors are on the host)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_30409_amd as gdn
from paper_2605_30409_amd import block

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN, ALIAS = -1, -2, -3, -4, -6, -7
BASE, MB = 1 << 40, 1 << 20


def addr(i):
    return BASE + i * 64 * MB


def test_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gdn_block.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(gdn_[a-z0-9_]+)\s*\(", src)))
    assert "gdn_gated_linear_forward" in names and "gdn_grad_clip" in names and len(names) == 10
    lib = ctypes.CDLL(gdn.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


FWD = dict(x=addr(0), w_gate=addr(1), w_up=addr(2), h=addr(3), M=100, C=72, F=40, act=1, bf16=1, ws=addr(4), ws_bytes=MB)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(w_gate=None), NULL), (dict(w_up=None), NULL), (dict(h=None), NULL), (dict(M=0), SHAPE), (dict(C=0), SHAPE),
    (dict(F=-1), SHAPE), (dict(C=1 << 21), SHAPE), (dict(F=1 << 20), SHAPE), (dict(M=1 << 30, F=1 << 19), SHAPE), (dict(act=4), UNSUPPORTED),
    (dict(act=-1), UNSUPPORTED), (dict(x=addr(0) + 8), ALIGN), (dict(h=addr(3) + 2), ALIGN), (dict(h=addr(0)), ALIAS), (dict(h=addr(1) + 16), ALIAS),
    (dict(C=71, ws=None), WORKSPACE), (dict(C=71, ws_bytes=100), WORKSPACE), (dict(C=71, ws=addr(4) + 16), WORKSPACE),
    (dict(C=71, ws=addr(0)), ALIAS), (dict(C=71, ws=addr(3)), ALIAS)])
def test_gated_refusals(kw, want):
    assert block._lib().gdn_gated_linear_forward(*dict(FWD, **kw).values(), None) == want


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("C,F", [(71, 40), (72, 41), (71, 41)])
def test_gated_alignment_is_that_of_the_rows(C, F, bf16):
    """Rows that are no whole multiples of 16 bytes start anywhere, and so may the tensor: the second half of one weight, say.  (What
    is taken is refused for h or dw_up, which are the same as another tensor, behind the check of alignment.)"""
    esz = 2 if bf16 else 4
    back = dict(x=addr(0), w_gate=addr(1), w_up=addr(2), dh=addr(3), dx=addr(4), dw_gate=addr(5), dw_up=addr(5), M=100, C=C, F=F, act=1, bf16=bf16,
                ws=addr(7), ws_bytes=16 * MB)
    fwd = dict(FWD, C=C, F=F, bf16=bf16, h=addr(0), ws_bytes=16 * MB)
    for args, call, names in ((fwd, block._lib().gdn_gated_linear_forward, ("x", "w_gate", "w_up", "h")),
                              (back, block._lib().gdn_gated_linear_backward, ("x", "w_gate", "w_up", "dh", "dx", "dw_gate", "dw_up"))):
        assert call(*args.values(), None) == ALIAS
        for name in names:
            loose = (F if name in ("h", "dh") else C) % 2 == 1
            for off, want in ((1, ALIGN), (esz // 2, ALIGN), (esz, ALIAS if loose else ALIGN), (8, ALIAS if loose else ALIGN)):
                assert call(*dict(args, **{name: args[name] + off}).values(), None) == want, (name, off)


BACK = dict(x=addr(0), w_gate=addr(1), w_up=addr(2), dh=addr(3), dx=addr(4), dw_gate=addr(5), dw_up=addr(6), M=100, C=72, F=40, act=1, bf16=1,
            ws=addr(7), ws_bytes=MB)


@pytest.mark.parametrize("kw", [dict(M=1 << 30, F=1 << 13), dict(M=1 << 30, C=1 << 13), dict(F=(1 << 20) - 1, C=(1 << 21) - 1)])
def test_gated_larger_than_a_launch(kw):
    a = dict(FWD, **kw)
    assert block._lib().gdn_gated_linear_forward(*a.values(), None) == SHAPE
    for backward in (0, 1):
        assert block._lib().gdn_gated_linear_workspace_bytes(a["M"], a["C"], a["F"], 1, backward) == 0
    assert block._lib().gdn_gated_linear_backward(*dict(BACK, **kw).values(), None) == SHAPE


@pytest.mark.parametrize("bf16", [0, 1])
def test_gated_copies_larger_than_a_launch(bf16):
    """Rows of odd length are copied first, 131080 threads each here: from 2^32 threads on the call is refused, where rows are copied."""
    fits, size = dict(C=(1 << 20) + 1, F=16350, bf16=bf16, ws_bytes=1 << 50), block._lib().gdn_gated_linear_workspace_bytes
    far = dict(x=(1 << 50) + 1, w_gate=1 << 51, w_up=1 << 52, ws=1 << 59)
    fwd, back = dict(FWD, h=1 << 53, **fits, **far), dict(BACK, dh=1 << 53, dx=1 << 54, dw_gate=1 << 55, dw_up=1 << 56, **fits, **far)
    for M, want in ((65, ALIGN), (66, SHAPE), (70, SHAPE)):
        assert block._lib().gdn_gated_linear_forward(*dict(fwd, M=M).values(), None) == want
        assert block._lib().gdn_gated_linear_backward(*dict(back, M=M).values(), None) == want
        for backward in (0, 1):
            assert (size(M, fits["C"], fits["F"], bf16, backward) == 0) == (want == SHAPE)
    more = dict(M=64, F=16352)                     # few rows are streamed as they are, but not for the gradient
    assert block._lib().gdn_gated_linear_forward(*dict(fwd, **more).values(), None) == ALIGN
    assert block._lib().gdn_gated_linear_backward(*dict(back, **more).values(), None) == SHAPE


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(w_gate=None), NULL), (dict(w_up=None), NULL), (dict(dh=None), NULL), (dict(dx=None), NULL),
    (dict(dw_gate=None), NULL), (dict(dw_up=None), NULL), (dict(M=0), SHAPE), (dict(F=0), SHAPE), (dict(act=9), UNSUPPORTED),
    (dict(dh=addr(3) + 4), ALIGN), (dict(dw_up=addr(6) + 8), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=addr(7) + 64), WORKSPACE),
    (dict(ws_bytes=1000), WORKSPACE), (dict(dx=addr(0)), ALIAS), (dict(dw_gate=addr(1)), ALIAS), (dict(dw_up=addr(5)), ALIAS),
    (dict(dx=addr(3)), ALIAS), (dict(ws=addr(2)), ALIAS), (dict(ws=addr(4)), ALIAS)])
def test_gated_gradient_refusals(kw, want):
    assert block._lib().gdn_gated_linear_backward(*dict(BACK, **kw).values(), None) == want


def test_gated_workspace():
    f = block._lib().gdn_gated_linear_workspace_bytes
    assert f(0, 8, 8, 1, 1) == 0 and f(8, 1 << 21, 8, 1, 1) == 0 and f(8, 8, 1 << 20, 1, 0) == 0
    assert f(10560, 2048, 8192, 1, 0) == 0 and f(1, 2048, 8192, 1, 0) == 0        # nothing but the outputs
    for M, C, F, bf16 in ((10560, 2048, 8192, 1), (333, 1283, 2711, 0), (1, 1, 1, 1), (64, 4096, 256, 1), (3520, 71, 65, 0)):
        esz, Fp = 2 if bf16 else 4, -(-F // 64) * 64
        ld = 0 if C * esz % 16 == 0 else -(-C // 64) * 64
        copies = (M + 2 * F) * ld * esz
        for backward in (0, 1):
            n = f(M, C, F, bf16, backward)
            need = copies + (2 * M * Fp * esz if backward else 0)
            # the sums of a contraction that is cut: no more than 512 tiles of 128 x 128, or 256 of 256 x 256, in fp32
            assert n <= need + 256 * 65536 * 4 + 2048
            if backward:
                assert n >= need


CONV = dict(x=addr(0), xb=1000, xt=100, w=addr(1), bias=addr(2), state_in=addr(3), y=addr(4), state_out=addr(5), B=2, T=10, C=40, W=4, act=1, bf16=1)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(y=None), NULL), (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(C=0), SHAPE),
    (dict(xt=-1), SHAPE), (dict(xb=-4), SHAPE), (dict(B=1 << 30, T=1 << 20), SHAPE), (dict(T=1 << 30), SHAPE), (dict(W=1), UNSUPPORTED),
    (dict(W=5), UNSUPPORTED), (dict(act=4), UNSUPPORTED), (dict(x=addr(0) + 1), ALIGN), (dict(w=addr(1) + 4), ALIGN), (dict(y=addr(4) + 2), ALIGN),
    (dict(y=addr(0)), ALIAS), (dict(y=addr(0) + 1600), ALIAS), (dict(y=addr(3)), ALIAS), (dict(state_out=addr(4)), ALIAS),
    (dict(state_out=addr(3) + 16), ALIAS), (dict(state_out=addr(2)), ALIAS), (dict(state_out=addr(0)), ALIAS)])
def test_conv_refusals(kw, want):
    assert block._lib().gdn_short_conv_forward(*dict(CONV, **kw).values(), None) == want


CGRAD = dict(x=addr(0), xb=1000, xt=100, w=addr(1), bias=addr(2), state_in=addr(3), dy=addr(4), dstate_out=addr(5), dx=addr(6), dxb=400, dxt=40,
             dw=addr(7), dbias=addr(8), dstate_in=addr(9), B=2, T=10, C=40, W=4, act=1, bf16=1, ws=addr(10), ws_bytes=MB)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(dy=None), NULL), (dict(dx=None), NULL), (dict(dw=None), NULL), (dict(T=0), SHAPE),
    (dict(dxt=39), SHAPE), (dict(dxb=399), SHAPE), (dict(dxt=-40), SHAPE), (dict(W=5), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(dx=addr(6) + 1), ALIGN), (dict(dy=addr(4) + 2), ALIGN), (dict(dw=addr(7) + 4), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=16), WORKSPACE),
    (dict(ws=addr(10) + 16), WORKSPACE), (dict(dx=addr(0)), ALIAS), (dict(dx=addr(4)), ALIAS), (dict(dw=addr(1)), ALIAS), (dict(dstate_in=addr(5)), ALIAS),
    (dict(dbias=addr(7)), ALIAS), (dict(ws=addr(0)), ALIAS), (dict(ws=addr(6)), ALIAS)])
def test_conv_gradient_refusals(kw, want):
    assert block._lib().gdn_short_conv_backward(*dict(CGRAD, **kw).values(), None) == want


@pytest.mark.parametrize("dxb,dxt,want", [(400, 40, None), (40, 80, None), (41, 81, None), (1000, 3000, None), (3000, 300, None), (39, 80, SHAPE),
                                          (40, 79, SHAPE), (400, 39, SHAPE), (399, 40, SHAPE), (0, 80, SHAPE), (40, 0, SHAPE), (-40, 80, SHAPE)])
def test_conv_gradient_layouts(dxb, dxt, want):
    """dx [2][10][40] with its sequences one behind the other, or all sequences of a token before the next token: any two strides that keep
    its elements apart.  (What is taken is refused for the workspace.)"""
    assert block._lib().gdn_short_conv_backward(*dict(CGRAD, dxb=dxb, dxt=dxt, ws=None).values(), None) == (want or WORKSPACE)


@pytest.mark.parametrize("B,T,dxb,dxt", [(1, 10, 0, 40), (2, 1, 40, 0), (1, 1, 0, 0)])
def test_conv_gradient_layouts_without_another_token_or_sequence(B, T, dxb, dxt):
    assert block._lib().gdn_short_conv_backward(*dict(CGRAD, B=B, T=T, dxb=dxb, dxt=dxt, ws=None).values(), None) == WORKSPACE


STEP = dict(x=addr(0), xb=1000, xt=100, w=addr(1), bias=addr(2), state_in=addr(3), slots=addr(4), lengths=addr(5), y=addr(6), state_out=addr(3), N=3,
            L=2, P=4, C=40, W=4, act=1, bf16=1)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(state_in=None), NULL), (dict(y=None), NULL), (dict(state_out=None), NULL), (dict(N=0), SHAPE),
    (dict(L=0), SHAPE), (dict(P=0), SHAPE), (dict(C=0), SHAPE), (dict(slots=None, N=5), SHAPE), (dict(N=1 << 20, C=1 << 14, P=1 << 20), SHAPE),
    (dict(W=5), UNSUPPORTED), (dict(act=7), UNSUPPORTED), (dict(slots=addr(4) + 2), ALIGN), (dict(lengths=addr(5) + 1), ALIGN), (dict(x=addr(0) + 1), ALIGN),
    (dict(state_in=addr(3) + 2), ALIGN), (dict(y=addr(0)), ALIAS), (dict(y=addr(3)), ALIAS), (dict(y=addr(4)), ALIAS), (dict(state_out=addr(3) + 16), ALIAS),
    (dict(state_out=addr(5)), ALIAS), (dict(state_out=addr(6)), ALIAS)])
def test_conv_step_refusals(kw, want):
    assert block._lib().gdn_short_conv_step(*dict(STEP, **kw).values(), None) == want


@pytest.mark.parametrize("kw", [dict(B=1 << 23, T=1, C=8), dict(B=1 << 20, T=1, C=2048), dict(B=1, T=1 << 29, C=8192)])
def test_conv_gradient_larger_than_a_launch(kw):
    kw = dict(kw, dx=1 << 60, x=1 << 50, dxt=kw["C"], dxb=kw["T"] * kw["C"])
    assert block._lib().gdn_short_conv_backward(*dict(CGRAD, **kw).values(), None) == SHAPE
    assert block._lib().gdn_short_conv_workspace_bytes(kw["B"], kw["T"], kw["C"], 4) == 0


def test_conv_larger_than_a_launch():
    """One token a sequence: a thread for 8 channels of each, so 512 threads a sequence here, and fewer than 2^32 in all.  (What is not
    refused for that is for its address.)"""
    args = dict(CONV, x=(1 << 50) + 1, xb=0, xt=0, y=1 << 60, state_in=None, state_out=None, T=1, C=4096)
    for B, want in (((1 << 23) - 1, ALIGN), (1 << 23, SHAPE), ((1 << 24) - 1, SHAPE)):
        assert block._lib().gdn_short_conv_forward(*dict(args, B=B).values(), None) == want


@pytest.mark.parametrize("W,C", [(4, 53687079), (3, 67108849), (2, 89478465)])
def test_conv_gradient_with_more_sums_than_a_launch(W, C):
    """(W + 1) C sums, 16 threads each in workgroups of 64 sums: from 2^32 threads on nothing is enqueued."""
    assert -(-(W + 1) * C // 64) == 1 << 22
    args = dict(CGRAD, x=(1 << 50) + 1, dx=1 << 51, dy=1 << 52, w=1 << 53, dw=1 << 54, bias=None, dbias=None, state_in=None, dstate_out=None,
                dstate_in=None, ws=1 << 55, ws_bytes=1 << 40, B=1, T=1, W=W)
    for c, want in ((C - 1, ALIGN), (C, SHAPE)):
        assert block._lib().gdn_short_conv_backward(*dict(args, C=c, dxt=c, dxb=c).values(), None) == want
        assert (block._lib().gdn_short_conv_workspace_bytes(1, 1, c, W) == 0) == (want == SHAPE)


def test_conv_workspace():
    f = block._lib().gdn_short_conv_workspace_bytes
    assert f(0, 1, 1, 4) == 0 and f(1, 1, 1, 5) == 0 and f(1, 1, 1, 1) == 0 and f(1 << 30, 1 << 20, 8, 4) == 0
    for B, T, C, W in ((1, 1, 1, 2), (1, 10560, 2048, 4), (70001, 2, 9, 3)):
        n = f(B, T, C, W)
        assert 0 < n <= (W + 1) * C * 4 * B * (T // 16 + 1) + 256


def arrays(tensors, sizes, kinds):
    n = len(tensors)
    return (ctypes.c_void_p * n)(*tensors), (ctypes.c_int64 * n)(*sizes), (ctypes.c_int * n)(*kinds)


def clip(tensors=(addr(0), addr(1)), out=(addr(2), addr(3)), sizes=(100, 50), kinds=(1, 0), count=2, norm_in=None, norm=addr(4), max_norm=1.0, eps=1e-6,
         ws=addr(5), ws_bytes=MB):
    t, s, k = arrays(tensors, sizes, kinds)
    o = (ctypes.c_void_p * len(out))(*out)
    return block._lib().gdn_grad_clip(t, o, s, k, count, norm_in, norm, max_norm, eps, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(count=-1), SHAPE), (dict(sizes=(100, -1)), SHAPE), (dict(sizes=(1 << 50, 1)), SHAPE), (dict(tensors=(None, addr(1))), NULL), (dict(out=(addr(2), None)), NULL),
    (dict(tensors=(addr(0) + 1, addr(1))), ALIGN), (dict(tensors=(addr(0), addr(1) + 2)), ALIGN), (dict(out=(addr(2), addr(3) + 2)), ALIGN),
    (dict(norm=addr(4) + 2), ALIGN), (dict(norm_in=addr(6) + 1), ALIGN), (dict(max_norm=-1.0), SHAPE), (dict(max_norm=float("nan")), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE), (dict(ws=addr(5) + 8), WORKSPACE),
    (dict(out=(addr(0), addr(0) + 100)), ALIAS), (dict(out=(addr(1), addr(3))), ALIAS), (dict(out=(addr(2), addr(2) + 196)), ALIAS),
    (dict(out=(addr(0) + 2, addr(3))), ALIAS), (dict(tensors=(addr(0), addr(0)), kinds=(1, 1), out=(addr(0), addr(0))), ALIAS),
    (dict(norm=addr(0)), ALIAS), (dict(norm=addr(2) + 4), ALIAS), (dict(norm=addr(5)), ALIAS), (dict(norm_in=addr(2)), ALIAS), (dict(ws=addr(0)), ALIAS),
    (dict(ws=addr(3)), ALIAS)])
def test_clip_refusals(kw, want):
    assert clip(**kw) == want


def test_norm_refusals():
    t, s, k = arrays((addr(0), addr(1)), (100, 50), (1, 0))
    f = block._lib().gdn_grad_norm
    assert f(t, s, k, 2, None, addr(5), MB, None) == NULL
    assert f(None, s, k, 2, addr(4), addr(5), MB, None) == NULL
    assert f(t, s, k, -1, addr(4), addr(5), MB, None) == SHAPE
    assert f(t, s, k, 2, addr(4) + 1, addr(5), MB, None) == ALIGN
    assert f(t, s, k, 2, addr(4), addr(5), 100, None) == WORKSPACE
    assert f(t, s, k, 2, addr(0), addr(5), MB, None) == ALIAS
    assert f(t, s, k, 2, addr(4), addr(1), MB, None) == ALIAS
    assert f(t, s, k, 2, addr(5) + 8, addr(5), MB, None) == ALIAS
    g = block._lib().gdn_grad_workspace_bytes
    assert g(-1) == 0 and 0 < g(0) <= g(1) == g(100) < g(1000)


def test_host_tensors_and_other_values_are_refused():
    """No fallback: a tensor that is not on a GPU is an error."""
    z = torch.zeros
    with pytest.raises(ValueError, match="GPU"):
        gdn.gated_linear(z(2, 8), z(4, 8), z(4, 8))
    with pytest.raises(TypeError, match="bfloat16"):
        gdn.gated_linear(z(2, 8).half(), z(4, 8), z(4, 8))
    with pytest.raises(TypeError, match="tensor"):
        gdn.gated_linear_backward(None, z(4, 8), z(4, 8), z(2, 4))
    with pytest.raises(ValueError, match="GPU"):
        gdn.short_conv(z(1, 2, 8), z(8, 4))
    with pytest.raises(ValueError, match="GPU"):
        gdn.short_conv_backward(z(1, 2, 8), z(8, 4), None, None, z(1, 2, 8))
    with pytest.raises(ValueError, match="GPU"):
        gdn.short_conv_step(z(1, 2, 8), z(8, 4), None, z(3, 3, 8))
    with pytest.raises(ValueError, match="GPU"):
        gdn.grad_norm([z(3)])
    with pytest.raises(ValueError, match="activation"):
        block._act("relu")
    with pytest.raises(ValueError, match="activation"):
        block._act(["silu"])
    for shape in ((1, 1 << 31, 8), (1 << 31, 1, 8)):
        with pytest.raises(ValueError, match="2.31"):
            gdn.short_conv_workspace(z(1, 1, 1).expand(*shape), z(8, 4))
    with pytest.raises(ValueError, match="2.31"):
        gdn.gated_linear_workspace(z(1, 1).expand(1 << 31, 8), z(4, 8))
    with pytest.raises(ValueError, match="unsupported"):
        gdn.short_conv_workspace(z(1, 2, 8), z(8, 5))
    assert gdn.gated_linear_workspace(z(200, 64), z(64, 64)).numel() == 0
    with pytest.raises(ValueError, match="no tensor"):
        gdn.grad_workspace([])


@pytest.mark.parametrize("shape,stride,dense", [((3, 4), (4, 1), True), ((3, 4), (1, 3), True), ((3, 4), (8, 1), False), ((3, 4), (4, 2), False),
                                                ((2, 3, 4), (4, 8, 1), True), ((1, 4), (100, 1), True), ((5,), (2,), False), ((2, 2), (0, 1), False)])
def test_tensors_that_fill_a_run_of_memory(shape, stride, dense):
    assert block._dense(torch.zeros(100).as_strided(shape, stride)) is dense
