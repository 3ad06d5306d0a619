"""The feed-forward and gradient operators' host side, without a GPU: what a
call refuses before any device work, and the scratch it asks for."""
import ctypes as C

import pytest

from paper_2609_34244_amd import heddle as H

P = 0x10000   # an address that no call below reads or writes


@pytest.fixture(scope="module")
def L():
    return H.lib()


def linear(**over):
    d = dict(dtype=H.HEDDLE_T_BF16, act=H.HEDDLE_A_SILU, m=100, n=64, k=96, x=P, ldx=96, w=P, ldw=96, residual=P, ldr=64,
             preact=P, ldp=64, y=P, ldy=64, dy=P, lddy=64, dx=P, lddx=96, dw=P, lddw=96, db=P, bias=P)
    d.update(over)
    return H.heddle_linear_desc(**d)


def ffn(**over):
    d = dict(dtype=H.HEDDLE_T_F16, act=H.HEDDLE_A_SILU, t=100, d=64, f=48, x=P, ldx=64, w_in=P, ldw_in=64, w_out=P, ldw_out=48,
             residual=P, ldr=64, preact=P, ldp=96, y=P, ldy=64, dy=P, lddy=64, dx=P, lddx=64, dw_in=P, lddw_in=64, dw_out=P,
             lddw_out=48)
    d.update(over)
    return H.heddle_gated_ffn_desc(**d)


def need(call, desc, backward):
    n = C.c_int64(-1)
    return call(C.byref(desc), backward, C.byref(n)), n.value


BOTH = [dict(dtype=H.HEDDLE_T_F32), dict(dtype=-1), dict(act=5), dict(act=-1), dict(d_offsets=P, groups=0),
        dict(d_offsets=P, groups=65536), dict(d_offsets=P + 2, groups=1)]
LINEAR = [dict(m=-1), dict(n=0), dict(k=0), dict(m=2**30 + 1), dict(n=2**22 + 1), dict(k=2**22 + 1)]
FFN = [dict(t=-1), dict(d=0), dict(f=0), dict(t=2**30 + 1), dict(d=2**22 + 1), dict(f=2**21 + 1)]
FORWARD = [dict(x=0), dict(x=P + 1), dict(ldx=0), dict(ldx=2**22 + 1), dict(y=0), dict(ldy=63), dict(ldr=63), dict(residual=P + 1),
           dict(preact=P + 1)]
BACKWARD = [dict(dy=0), dict(lddy=63), dict(preact=0), dict(ldp=63), dict(dx=P + 1), dict(lddx=1), dict(x=0), dict(ldx=-1)]


@pytest.mark.parametrize("over", BOTH + LINEAR + FORWARD + [dict(w=0), dict(ldw=95), dict(bias=P + 1),
                                                            dict(d_offsets=P, groups=2, stride_w=63 * 96 + 95)])
def test_linear_refuses(L, over):
    d = linear(**over)
    assert need(L.heddle_linear_workspace, d, 0)[0] == H.HEDDLE_E_INVAL and H.heddle_last_error()
    assert L.heddle_linear(C.byref(d), None, 0, None) == H.HEDDLE_E_INVAL


@pytest.mark.parametrize("over", BOTH + LINEAR + BACKWARD + [dict(w=0), dict(lddw=95), dict(db=P + 1),
                                                             dict(d_offsets=P, groups=2, stride_w=2**20, stride_dw=6143)])
def test_linear_backward_refuses(L, over):
    d = linear(**over)
    assert need(L.heddle_linear_workspace, d, 1)[0] == H.HEDDLE_E_INVAL
    assert L.heddle_linear_backward(C.byref(d), None, 0, None) == H.HEDDLE_E_INVAL


@pytest.mark.parametrize("over", BOTH + FFN + FORWARD + [dict(w_in=0), dict(w_out=0), dict(ldw_out=47),
                                                         dict(d_offsets=P, groups=2, stride_in=1, stride_out=2**20)])
def test_ffn_refuses(L, over):
    d = ffn(**over)
    assert need(L.heddle_gated_ffn_workspace, d, 0)[0] == H.HEDDLE_E_INVAL and H.heddle_last_error()
    assert L.heddle_gated_ffn(C.byref(d), None, 0, None) == H.HEDDLE_E_INVAL


@pytest.mark.parametrize("over", BOTH + FFN + BACKWARD + [dict(w_in=0), dict(w_out=0), dict(lddw_in=63), dict(lddw_out=47),
                                                          dict(d_offsets=P, groups=2, stride_in=2**20, stride_out=2**20,
                                                               stride_dw_in=2**20, stride_dw_out=1)])
def test_ffn_backward_refuses(L, over):
    d = ffn(**over)
    assert need(L.heddle_gated_ffn_workspace, d, 1)[0] == H.HEDDLE_E_INVAL
    assert L.heddle_gated_ffn_backward(C.byref(d), None, 0, None) == H.HEDDLE_E_INVAL


def test_workspace(L):
    """what a call needs is told without a device, and less of it is refused"""
    for call, work, desc, backward in ((L.heddle_linear_workspace, L.heddle_linear_backward, linear(), 1),
                                       (L.heddle_gated_ffn_workspace, L.heddle_gated_ffn, ffn(), 0),
                                       (L.heddle_gated_ffn_workspace, L.heddle_gated_ffn_backward, ffn(), 1)):
        rc, n = need(call, desc, backward)
        assert rc == H.HEDDLE_OK and n >= 100 * 48 * 2
        assert work(C.byref(desc), P, n - 1, None) == H.HEDDLE_E_INVAL
        assert work(C.byref(desc), P + 128, n, None) == H.HEDDLE_E_INVAL and "256" in H.heddle_last_error()
        assert work(C.byref(desc), None, n, None) == H.HEDDLE_E_INVAL
        assert call(C.byref(desc), backward, None) == H.HEDDLE_E_INVAL
        assert call(None, backward, C.byref(C.c_int64())) == H.HEDDLE_E_INVAL and work(None, P, n, None) == H.HEDDLE_E_INVAL


def test_one_group_needs_no_more_than_its_copies(L):
    """with offsets a reduction is not divided, so there are no parts to keep, also for one group"""
    long = dict(m=20000, act=H.HEDDLE_A_NONE, db=0)
    assert need(L.heddle_linear_workspace, linear(**long), 1)[1] > 0
    assert need(L.heddle_linear_workspace, linear(d_offsets=P, groups=1, **long), 1)[1] == 0


def test_clipping_refuses(L):
    def grads(**over):
        d = dict(g=P, out=P, n=10, dtype=H.HEDDLE_T_F32)
        d.update(over)
        return H.heddle_grad_desc(**d)

    def calls(g, count, max_norm=1.0, norm=P, ws=P, n=1 << 20):
        return [L.heddle_grad_norm(g, count, norm, ws, n, None), L.heddle_clip_grad_norm(g, count, max_norm, norm, ws, n, None),
                L.heddle_clip_grads(g, count, norm, max_norm, None)]

    for over in (dict(g=0), dict(g=P + 2), dict(out=P + 2), dict(n=-1), dict(n=2**40 + 1), dict(dtype=3)):
        assert calls(C.byref(grads(**over)), 1) == [H.HEDDLE_E_INVAL] * 3, over
    one = C.byref(grads())
    assert calls(one, -1) == calls(None, 1) == calls(one, 1, norm=P + 2) == calls(one, 1, norm=None) == [H.HEDDLE_E_INVAL] * 3
    for over in (dict(ws=None), dict(ws=P + 8), dict(n=8)):
        assert calls(None, 0, max_norm=0.0, **over) == [H.HEDDLE_E_INVAL] * 3
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert calls(one, 1, max_norm=bad, ws=None) == [H.HEDDLE_E_INVAL] * 3
    n = C.c_int64()
    assert L.heddle_grad_norm_workspace(one, 1, C.byref(n)) == H.HEDDLE_OK and n.value >= 8
    assert L.heddle_grad_norm_workspace(one, 1, None) == H.HEDDLE_E_INVAL
