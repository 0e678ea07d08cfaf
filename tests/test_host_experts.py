"""Refusals of the experts' entry points, on the host: nothing below reaches
a device."""
import ctypes

import pytest

from paper_2609_36959_amd import binding as B

EINVAL, EUNSUPPORTED = 1, 2
P = ctypes.c_void_p
OK = P(4096)       # never dereferenced
ODD = P(4104)      # not 16-byte aligned
BIG = 1 << 40


def call(name, *args):
    return getattr(B.lib(), name)(*args)


def test_group():
    def group(topk=OK, pos=None, T=8, K=2, E=4, rows=OK, off=OK, ws=OK, n=BIG):
        return call("cobalt_expert_group", topk, pos, T, K, E, rows, None, off, ws, n, None)
    assert group(topk=None) == group(rows=None) == group(off=None) == group(ws=None) == EINVAL
    assert group(T=-1) == group(K=0) == group(K=17) == group(E=0) == group(E=4097) == EINVAL
    assert group(ws=ODD) == group(n=16) == EINVAL
    assert group(T=1 << 30) == EUNSUPPORTED
    size = B.cobalt_expert_group_workspace_bytes
    assert size(-1, 2, 4) == size(8, 17, 4) == size(8, 2, 4097) == size(1 << 30, 2, 4) == 0
    last = 0
    for T in (0, 1, 1000, 10**4, 10**5, 10**6, 10**8):
        assert size(T, 8, 64) >= last and size(T, 8, 65) >= size(T, 8, 64) > 0
        last = size(T, 8, 64)


SIZES = dict(M=8, E=4, d=16, f=16)


def sizes(unit):
    """Sizes that every product refuses, and with what."""
    yield dict(M=-1), EINVAL
    yield dict(E=0), EINVAL
    yield dict(E=4097), EINVAL
    yield dict(d=0), EINVAL
    yield dict(f=0), EINVAL
    yield dict(d=unit + 4), EINVAL
    yield dict(f=unit + 4), EINVAL
    yield dict(M=1 << 31), EUNSUPPORTED
    yield dict(d=(1 << 20) + unit), EUNSUPPORTED
    yield dict(f=(1 << 20) + unit), EUNSUPPORTED


def gate_up(x=OK, n=8, rows=OK, off=OK, M=8, E=4, d=16, f=16, w=OK, act=0, h=OK, gu=None):
    return call("cobalt_expert_gate_up", x, n, rows, off, M, E, d, f, w, act, h, gu, None)


def down(h=OK, off=OK, M=8, E=4, d=16, f=16, w=OK, rows=OK, n=8, out=OK):
    return call("cobalt_expert_down", h, off, M, E, d, f, w, rows, n, out, None)


def down_backward(dout=OK, n=8, rows=OK, off=OK, M=8, E=4, d=16, f=16, w=OK, gu=OK, h=OK, act=0,
                  dgu=OK, dw=OK, flags=0, ws=OK, size=BIG):
    return call("cobalt_expert_down_backward", dout, n, rows, off, M, E, d, f, w, gu, h, act, dgu,
                dw, flags, ws, size, None)


def gate_up_backward(dgu=OK, x=OK, n=8, rows=OK, off=OK, M=8, E=4, d=16, f=16, w=OK, dx=OK, dw=OK,
                     flags=0, ws=OK, size=BIG):
    return call("cobalt_expert_gate_up_backward", dgu, x, n, rows, off, M, E, d, f, w, dx, dw,
                flags, ws, size, None)


def mx_gate_up(x=OK, xs=OK, n=8, rows=OK, off=OK, M=8, E=4, d=32, f=32, w=OK, ws=OK, act=0, h=OK):
    return call("cobalt_mx_gate_up", x, xs, n, rows, off, M, E, d, f, w, ws, act, h, None)


def mx_down(h=OK, hs=OK, off=OK, M=8, E=4, d=32, f=32, w=OK, ws=OK, rows=OK, n=8, out=OK):
    return call("cobalt_mx_down", h, hs, off, M, E, d, f, w, ws, rows, n, out, None)


@pytest.mark.parametrize("fn,unit", [(gate_up, 8), (down, 8), (down_backward, 8),
                                     (gate_up_backward, 8), (mx_gate_up, 32), (mx_down, 32)])
def test_sizes(fn, unit):
    for bad, status in sizes(unit):
        assert fn(**{"n": 1 << 33, **bad}) == status, bad
    assert fn(off=None) == fn(n=-1) == EINVAL
    assert fn(rows=None, n=7) == EINVAL          # places without a row of their own
    assert fn(w=None) == fn(w=ODD) == EINVAL


def test_buffers():
    assert gate_up(x=None) == gate_up(x=ODD) == gate_up(h=None) == gate_up(h=ODD) == EINVAL
    assert gate_up(gu=ODD) == gate_up(act=2) == gate_up(act=-1) == EINVAL
    assert down(h=None) == down(h=ODD) == down(out=None) == down(out=ODD) == EINVAL
    for b in (down_backward, gate_up_backward):
        assert b(flags=2) == b(flags=4) == b(flags=-1) == EINVAL
        assert b(ws=None) == b(ws=P(4096 + 16)) == b(size=255) == b(dw=ODD) == EINVAL
    assert down_backward(dout=None) == down_backward(gu=None) == down_backward(h=None) == EINVAL
    assert down_backward(dgu=ODD) == down_backward(gu=ODD) == down_backward(act=2) == EINVAL
    assert gate_up_backward(dgu=None) == gate_up_backward(x=None) == EINVAL
    assert gate_up_backward(dx=ODD) == gate_up_backward(x=ODD) == EINVAL
    assert mx_gate_up(x=None) == mx_gate_up(xs=None) == mx_gate_up(ws=None) == EINVAL
    assert mx_gate_up(x=ODD) == mx_gate_up(h=ODD) == mx_gate_up(act=3) == EINVAL
    assert mx_down(h=None) == mx_down(hs=None) == mx_down(ws=None) == mx_down(out=ODD) == EINVAL


def test_nothing_to_do():
    assert gate_up(M=0, n=0, x=None, h=None) == 0
    assert down(M=0, n=0, h=None, out=None) == 0
    assert down(n=0, out=None) == 0
    assert down_backward(M=0, n=0, dout=None, gu=None, h=None, dw=None) == 0
    assert gate_up_backward(dx=None, dw=None) == 0
    assert mx_gate_up(M=0, n=0, x=None, xs=None, h=None) == 0
    assert mx_down(n=0, out=None) == 0


def test_quantize():
    def quantize(x=OK, R=4, n=64, q=OK, s=OK):
        return (call("cobalt_mx_quantize", x, R, n, q, s, None),
                call("cobalt_mx_dequantize", q, s, R, n, x, None))
    for bad in (dict(x=None), dict(x=ODD), dict(q=None), dict(q=ODD), dict(s=None), dict(R=-1),
                dict(n=0), dict(n=48), dict(n=-32)):
        assert quantize(**bad) == (EINVAL, EINVAL), bad
    assert quantize(R=1 << 42, n=64) == (EUNSUPPORTED, EUNSUPPORTED)
    assert quantize(x=None, q=None, s=None, R=0) == (0, 0)


def test_combine_backward():
    def grad(dy=OK, eo=OK, pos=OK, gates=OK, T=8, K=2, d=16, deo=OK, dg=OK):
        return call("cobalt_combine_backward", dy, eo, pos, gates, T, K, d, deo, dg, None)
    for bad in (dict(dy=None), dict(dy=ODD), dict(eo=None), dict(eo=ODD), dict(pos=None),
                dict(gates=None), dict(deo=ODD), dict(T=-1), dict(K=0), dict(K=17), dict(d=12),
                dict(d=0)):
        assert grad(**bad) == EINVAL, bad
    assert grad(T=1 << 30) == EUNSUPPORTED
    assert grad(T=0, dy=None, eo=None, pos=None, gates=None) == 0
    assert grad(deo=None, dg=None) == 0


def test_backward_workspace():
    size = B.cobalt_expert_backward_workspace_bytes
    assert size(8, 4, 16, 16) >= 256
    assert size(-1, 4, 16, 16) == size(8, 0, 16, 16) == size(8, 4, 12, 16) == size(8, 4, 16, 0) == 0


def test_backward_workspace_grows_with_places():
    size = B.cobalt_expert_backward_workspace_bytes
    for E, d, f in ((1, 64, 32), (4, 512, 256), (8, 1024, 512), (64, 2048, 1024)):
        sizes = [size(M, E, d, f) for M in (0, 1, 500, 4096, 5000, 16384, 100000, 2**31 - 512)]
        assert sizes == sorted(sizes) and sizes[0] == 256
