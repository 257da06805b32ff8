"""Host-side checks of the operators in gdn_ops.h: exported symbols, workspace sizes and
refused arguments (no kernel is launched: addresses are made up, or the tensors
are on the host)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_30409_amd as gdn
from paper_2605_30409_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN, ALIAS = -1, -2, -3, -4, -6, -7
BASE, MB = 1 << 40, 1 << 20


def test_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gdn_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(gdn_[a-z0-9_]+)\s*\(", src)))
    assert "gdn_step_forward" in names and "gdn_block_norm_backward" in names
    lib = ctypes.CDLL(gdn.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def addr(i):
    return BASE + i * 64 * MB


STEP = dict(q=addr(0), k=addr(1), v=addr(2), alpha=addr(3), beta=addr(4), state_in=addr(5), slots=addr(6),
            lengths=addr(7), out=addr(8), state_out=addr(9), N=3, L=2, P=4, Hk=2, H=4, Dk=64, Dv=128, bf16=1)


def step(**kw):
    a = dict(STEP, **kw)
    return ops._lib().gdn_step_forward(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(alpha=None), NULL),
    (dict(beta=None), NULL), (dict(state_in=None), NULL), (dict(out=None), NULL), (dict(state_out=None), NULL),
    (dict(N=0), SHAPE), (dict(L=0), SHAPE), (dict(P=0), SHAPE), (dict(Hk=0), SHAPE), (dict(H=0), SHAPE),
    (dict(H=3), SHAPE), (dict(N=-1), SHAPE), (dict(slots=None, N=5), SHAPE), (dict(N=1 << 20, H=1 << 12), SHAPE),
    (dict(Dk=96), UNSUPPORTED), (dict(Dv=32), UNSUPPORTED),
    (dict(q=addr(0) + 8), ALIGN), (dict(state_out=addr(9) + 4), ALIGN), (dict(slots=addr(6) + 2), ALIGN),
    (dict(lengths=addr(7) + 1), ALIGN),
    (dict(out=addr(2)), ALIAS), (dict(out=addr(5)), ALIAS), (dict(out=addr(6)), ALIAS), (dict(state_out=addr(8)), ALIAS),
    (dict(state_out=addr(5) + 16), ALIAS), (dict(state_out=addr(0)), ALIAS), (dict(state_out=addr(7)), ALIAS)])
def test_step_refusals(kw, want):
    assert step(**kw) == want


NORM = dict(x=addr(0), y=addr(1), gate=addr(2), w_post=addr(3), w_pre=addr(4), r=addr(5), u=addr(6), R=12, C=40, gt=4,
            rs=1.0, eps=1e-6, bf16=1)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(w_post=None), NULL), (dict(w_pre=None), NULL), (dict(r=None), NULL),
    (dict(u=None), NULL), (dict(R=0), SHAPE), (dict(C=0), SHAPE), (dict(gt=0), SHAPE), (dict(gt=5), SHAPE),
    (dict(C=8193), UNSUPPORTED), (dict(x=addr(0) + 2), ALIGN), (dict(gate=addr(2) + 8), ALIGN),
    (dict(r=addr(6)), ALIAS), (dict(u=addr(0)), ALIAS), (dict(r=addr(0) + 16), ALIAS), (dict(u=addr(1) + 16), ALIAS),
    (dict(r=addr(2)), ALIAS), (dict(u=addr(3)), ALIAS)])
def test_norm_refusals(kw, want):
    assert ops._lib().gdn_block_norm_forward(*dict(NORM, **kw).values(), None) == want


GRAD = dict(x=addr(0), y=addr(1), gate=addr(2), w_post=addr(3), w_pre=addr(4), du=addr(5), dr=addr(6), dx=addr(7),
            dy=addr(8), dgate=addr(9), dw_post=addr(10), dw_pre=addr(11), R=12, C=40, gt=4, rs=1.0, eps=1e-6, bf16=1,
            ws=addr(12), ws_bytes=MB)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(du=None), NULL), (dict(dx=None), NULL), (dict(dw_pre=None), NULL),
    (dict(gate=None), NULL), (dict(dgate=None), NULL), (dict(R=13), SHAPE), (dict(C=9000), UNSUPPORTED),
    (dict(dy=addr(8) + 8), ALIGN), (dict(dr=addr(6) + 4), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(ws=addr(12) + 128), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE), (dict(dx=addr(0)), ALIAS),
    (dict(dx=addr(1)), ALIAS), (dict(dy=addr(0)), ALIAS), (dict(dx=addr(8)), ALIAS), (dict(dgate=addr(2)), ALIAS),
    (dict(dw_pre=addr(10)), ALIAS), (dict(ws=addr(5)), ALIAS), (dict(ws=addr(11)), ALIAS),
    (dict(dx=addr(5) + 16), ALIAS)])
def test_norm_gradient_refusals(kw, want):
    assert ops._lib().gdn_block_norm_backward(*dict(GRAD, **kw).values(), None) == want


@pytest.mark.parametrize("kw", [dict(N=1 << 13, H=1 << 11, P=1 << 13), dict(N=1 << 24, H=1, Hk=1, P=1 << 24)])
def test_step_larger_than_a_launch(kw):
    assert step(**dict(dict(out=1 << 60, state_out=addr(5)), **kw)) == SHAPE


@pytest.mark.parametrize("B,H,T", [(1, 1, 1 << 30), (8, 64, 1 << 20), (1, 65535, 129 * 64)])
def test_backward_larger_than_a_launch(B, H, T):
    assert ops._lib().gdn_chunk_backward_workspace_bytes(B, H, T, 64, 64, 64, 1) == 0
    assert ops._lib().gdn_chunk_backward(*dict(BACK, B=B, H=H, T=T).values(), None) == SHAPE


def test_norm_workspace():
    f = ops._lib().gdn_block_norm_workspace_bytes
    assert f(12, 40, 5) == 0 and f(0, 40, 1) == 0 and f(12, 8193, 1) == 0
    for R, C, gt in ((1, 1, 1), (12, 40, 4), (10560, 2048, 3520), (100000, 8, 1), (99999, 16, 3), (700, 64, 700)):
        n = f(R, C, gt)
        team = 64
        while 8 * team < C:
            team *= 2
        rows = -(-R // max(512, (1 << 17) // team))
        assert 0 < n <= 12 * C * (R // max(1, min(rows, gt)) + R // gt + 1) + 1024


def test_host_tensors_are_refused():
    """No fallback: a tensor that is not on a GPU is an error."""
    z = torch.zeros
    q, v = z(1, 1, 2, 64), z(1, 1, 2, 64)
    with pytest.raises(ValueError, match="GPU"):
        gdn.step(q, q, v, z(1, 1, 2), z(1, 1, 2), z(1, 2, 64, 64))
    with pytest.raises(TypeError, match="bfloat16"):
        gdn.step(q.half(), q, v, z(1, 1, 2), z(1, 1, 2), z(1, 2, 64, 64))
    with pytest.raises(ValueError, match="GPU"):
        gdn.block_norm(z(1, 2, 8), z(1, 2, 8), None, z(8), z(8))
    with pytest.raises(ValueError, match="GPU"):
        gdn.block_norm_backward(z(1, 2, 8), z(1, 2, 8), None, z(8), z(8), z(1, 2, 8))
    with pytest.raises(TypeError, match="tensor"):
        gdn.block_norm([1.0], z(1, 2, 8), None, z(8), z(8))


BACK = dict(q=addr(0), k=addr(1), v=addr(2), alpha=addr(3), beta=addr(4), state_in=addr(5), dout=addr(6),
            dstate_out=addr(7), dq=addr(8), dk=addr(9), dv=addr(10), dalpha=addr(11), dbeta=addr(12), dstate_in=addr(13),
            B=1, H=2, T=100, Dk=64, Dv=128, chunk=64, bf16=1, ws=addr(14), ws_bytes=32 * MB)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(alpha=None), NULL), (dict(beta=None), NULL),
    (dict(dout=None), NULL), (dict(dq=None), NULL), (dict(dk=None), NULL), (dict(dv=None), NULL),
    (dict(dalpha=None), NULL), (dict(dbeta=None), NULL), (dict(B=0), SHAPE), (dict(H=0), SHAPE), (dict(T=0), SHAPE),
    (dict(B=300, H=300), SHAPE), (dict(B=1, H=65535, T=1 << 30), SHAPE), (dict(Dk=96), UNSUPPORTED),
    (dict(Dv=256), UNSUPPORTED), (dict(chunk=32), UNSUPPORTED), (dict(dout=addr(6) + 8), ALIGN),
    (dict(dstate_in=addr(13) + 4), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=addr(14) + 16), WORKSPACE),
    (dict(ws_bytes=4096), WORKSPACE), (dict(dq=addr(0)), ALIAS), (dict(dv=addr(6)), ALIAS), (dict(dk=addr(8)), ALIAS),
    (dict(dalpha=addr(3)), ALIAS), (dict(dstate_in=addr(7) + 16), ALIAS), (dict(dstate_in=addr(5)), ALIAS),
    (dict(ws=addr(2)), ALIAS), (dict(ws=addr(10)), ALIAS)])
def test_backward_refusals(kw, want):
    assert ops._lib().gdn_chunk_backward(*dict(BACK, **kw).values(), None) == want


def test_backward_workspace():
    f = ops._lib().gdn_chunk_backward_workspace_bytes
    assert f(1, 2, 100, 96, 64, 64, 1) == 0 and f(1, 2, 0, 64, 64, 64, 1) == 0 and f(1, 2, 100, 64, 64, 32, 1) == 0
    n = 16 * 55
    per = 4 * (400 + 64 * 128 + 3 * 128 * 128 + 2 * 64 * 128)       # gates, N0, C0 and states, e and dV
    for bf16, planes in ((1, 6), (0, 4)):
        want = n * (per + 2 * planes * 64 * 64)
        assert want <= f(1, 16, 3520, 128, 128, 64, bf16) < want + 12 * 256
    with pytest.raises(ValueError, match="unsupported"):
        gdn.backward_workspace(torch.zeros(1, 3, 2, 32), torch.zeros(1, 3, 2, 64))


@pytest.mark.parametrize("rows,channels,gate_tokens", [((1 << 32) + 12, 40, 4), (12, (1 << 32) + 40, 4), (12, 40, (1 << 32) + 4),
                                                       (12, 40, 4.5), (12.5, 40, 1), (-12, 40, 4)])
def test_norm_workspace_of_sizes_past_32_bits(rows, channels, gate_tokens):
    """Sizes that 32 bits or whole numbers do not hold are refused, not cut to others."""
    with pytest.raises(ValueError):
        gdn.block_norm_workspace(rows, channels, gate_tokens, "cpu")
    assert gdn.block_norm_workspace(12.0, 40, 4, "cpu").numel() == gdn.block_norm_workspace(12, 40, 4, "cpu").numel()


def test_backward_workspace_of_sizes_past_32_bits():
    one = torch.zeros(1, 1, 1, 64)
    for shape in ((1, (1 << 32) + 100, 2), ((1 << 32) + 1, 100, 2), (1, 100, (1 << 32) + 2)):
        q = one.expand(*shape, 64)
        with pytest.raises(ValueError):
            gdn.backward_workspace(q, q)
    for chunk in ((1 << 32) + 64, 64.5):
        with pytest.raises(ValueError):
            gdn.backward_workspace(torch.zeros(1, 100, 2, 64), torch.zeros(1, 100, 2, 64), chunk)
