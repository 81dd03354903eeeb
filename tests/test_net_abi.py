"""Host-side refusals of the layers, norms and losses of a population of networks
(validation runs before any HIP call, so no GPU is needed)."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def evox():
    import paper_2301_12457_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2301_12457_amd import build
        build.build()
    return m


P = 0x1000  # never dereferenced


def layer(evox, **kw):
    d = dict(dtype=evox.F32, act=0, G=2, M=6, n_in=4, n_out=3, off=None, x_shared=0, ldx=4, ldw=4, w_stride=12,
             b_stride=3, ldr=3, ldz=3, ldy=3, lddx=4, lddw=4, dw_stride=12, db_stride=3)
    d.update(kw)
    return evox.Layer(**d)


def linear(evox, l, x=P, w=P, b=None, r=None, z=None, y=P):
    return evox.lib().evox_linear(ctypes.byref(l) if l else None, x, w, b, r, z, y, None)


def linear_grad(evox, l, x=P, w=P, z=P, dy=P, dx=P, dw=P, db=P, scratch=P, nbytes=1 << 40):
    return evox.lib().evox_linear_grad(ctypes.byref(l), x, w, z, dy, dx, dw, db, scratch, nbytes, None)


def test_struct_layouts(evox):
    assert ctypes.sizeof(evox.Layer) == 8 + 4 * 8 + 8 + 8 + 11 * 8
    assert evox.Layer.off.offset == 40 and evox.Layer.ldx.offset == 56
    assert ctypes.sizeof(evox.Norm) == 8 + 3 * 8 + 8 + 5 * 8 + 8 and evox.Norm.off.offset == 32
    assert ctypes.sizeof(evox.Classes) == 8 + 3 * 8 + 8 + 8 + 16 and evox.Classes.ldz.offset == 48


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(act=5), dict(act=-1), dict(G=0), dict(G=4),
                                dict(G=1 << 21, M=0), dict(M=-1), dict(M=1 << 31), dict(n_in=0), dict(n_out=0),
                                dict(n_in=1 << 21), dict(ldx=3), dict(ldw=3), dict(ldy=2), dict(w_stride=11),
                                dict(w_stride=-12), dict(w_stride=1 << 41), dict(ldx=1 << 45), dict(off=P, x_shared=1)])
def test_linear_refuses(evox, kw):
    assert linear(evox, layer(evox, **kw)) == evox.EINVAL
    assert len(evox.lib().evox_last_error()) > 5


def test_linear_refuses_operands(evox):
    l = layer(evox)
    assert linear(evox, None) == evox.EINVAL
    for k in ("x", "w", "y"):
        assert linear(evox, l, **{k: None}) == evox.EINVAL
    for k in ("x", "w", "b", "r", "z", "y"):
        assert linear(evox, l, **{k: P + 2}) == evox.EALIGN
        assert linear(evox, layer(evox, dtype=evox.BF16), **{k: P + 1}) == evox.EALIGN
    assert linear(evox, layer(evox, off=P + 2)) == evox.EALIGN
    assert linear(evox, layer(evox, b_stride=2), b=P) == evox.EINVAL
    assert linear(evox, layer(evox, ldr=2), r=P) == evox.EINVAL
    assert linear(evox, layer(evox, ldz=2), z=P) == evox.EINVAL
    assert linear(evox, layer(evox, M=0), x=None, w=None, y=None) == evox.OK  # nothing to do


def test_linear_grad_refuses(evox):
    g = lambda **kw: layer(evox, act=evox.ACT_TANH, **kw)
    need = evox.lib().evox_linear_grad_scratch_bytes(ctypes.byref(g()))
    assert need > 0 and evox.lib().evox_linear_grad_scratch_bytes(ctypes.byref(g(n_in=0))) == 0
    for k in ("x", "w", "z", "dy"):
        assert linear_grad(evox, g(), **{k: None}) == evox.EINVAL
    for k in ("x", "w", "z", "dy", "dx", "dw", "db"):
        assert linear_grad(evox, g(), **{k: P + 2}) == evox.EALIGN
    for kw in (dict(x_shared=1), dict(w_stride=0), dict(dw_stride=11), dict(db_stride=2), dict(lddx=3), dict(lddw=3),
               dict(ldz=2), dict(ldy=2)):
        assert linear_grad(evox, g(**kw)) == evox.EINVAL, kw
    assert linear_grad(evox, g(), scratch=None) == evox.EINVAL
    assert linear_grad(evox, g(), scratch=P + 16) == evox.EALIGN
    assert linear_grad(evox, g(), nbytes=need - 1) == evox.ENOSPC


def norm(evox, **kw):
    d = dict(dtype=evox.F32, G=2, M=6, D=5, off=None, ldx=5, ldy=5, lddx=5, p_stride=5, dp_stride=5, eps=1e-5)
    d.update(kw)
    return evox.Norm(**d)


def test_norm_refuses(evox):
    L = evox.lib()
    f = lambda n, x=P, ga=P, be=P, y=P, m=P, r=P: L.evox_layernorm(ctypes.byref(n), x, ga, be, y, m, r, None)
    for kw in (dict(dtype=9), dict(G=4), dict(D=0), dict(D=32769), dict(ldx=4), dict(ldy=4), dict(p_stride=4),
               dict(eps=0.0), dict(eps=float("nan"))):
        assert f(norm(evox, **kw)) == evox.EINVAL, kw
    for k in ("x", "ga", "be", "y"):
        assert f(norm(evox), **{k: None}) == evox.EINVAL
        assert f(norm(evox), **{k: P + 2}) == evox.EALIGN
    assert f(norm(evox), m=P + 2) == evox.EALIGN
    b = lambda n, x=P, ga=P, m=P, r=P, dy=P, dx=P, dg=P, db=P, s=P, nb=1 << 40: L.evox_layernorm_grad(
        ctypes.byref(n), x, ga, m, r, dy, dx, dg, db, s, nb, None)
    for kw in (dict(lddx=4), dict(dp_stride=4), dict(p_stride=0), dict(dp_stride=0)):
        assert b(norm(evox, **kw)) == evox.EINVAL, kw
    for k in ("x", "ga", "m", "r", "dy", "dg", "s"):
        assert b(norm(evox), **{k: None}) == evox.EINVAL
    need = L.evox_layernorm_grad_scratch_bytes(ctypes.byref(norm(evox)))
    assert need > 0 and L.evox_layernorm_grad_scratch_bytes(ctypes.byref(norm(evox, D=0))) == 0
    assert b(norm(evox), nb=need - 1) == evox.ENOSPC


def test_xent_refuses(evox):
    L = evox.lib()

    def classes(**kw):
        d = dict(dtype=evox.F32, G=2, M=6, C=5, off=None, labels_shared=0, ldz=5, lddz=5)
        d.update(kw)
        return evox.Classes(**d)

    f = lambda c, z=P, lab=P, fit=P, dz=P, s=P, nb=1 << 40: L.evox_xent(ctypes.byref(c), z, lab, fit, dz, s, nb, None)
    for kw in (dict(dtype=9), dict(G=4), dict(C=0), dict(C=32769), dict(ldz=4), dict(lddz=4), dict(off=P, labels_shared=1)):
        assert f(classes(**kw)) == evox.EINVAL, kw
    for k in ("z", "lab", "fit", "s"):
        assert f(classes(), **{k: None}) == evox.EINVAL
    for k in ("z", "lab", "fit", "dz"):
        assert f(classes(), **{k: P + 2}) == evox.EALIGN
    need = L.evox_xent_scratch_bytes(ctypes.byref(classes()))
    assert need > 0 and f(classes(), nb=need - 1) == evox.ENOSPC


def test_binding_refuses(evox):
    x, w, y = torch.zeros(6, 4), torch.zeros(2, 3, 4), torch.zeros(6, 3)
    bad = [dict(x=x.double()), dict(x=x[:5]), dict(x=torch.zeros(6, 8)[:, ::2]), dict(w=w[0]), dict(w=w.transpose(1, 2)),
           dict(y=y.bfloat16()), dict(b=torch.zeros(3)), dict(r=torch.zeros(6, 4)), dict(z=torch.zeros(5, 3)),
           dict(off=torch.zeros(3)), dict(off=torch.zeros(2, dtype=torch.int32))]
    for kw in bad:
        with pytest.raises(evox.EvoxError):
            evox.evox_linear(**dict(dict(x=x, w=w, y=y), **kw))
    p, st = torch.zeros(2, 4), torch.zeros(6)
    with pytest.raises(evox.EvoxError):
        evox.evox_layernorm(x, p, p[:, :3], x)
    with pytest.raises(evox.EvoxError):
        evox.evox_layernorm(x, p, p, x, mean=st.double())
    with pytest.raises(evox.EvoxError):
        evox.evox_layernorm_grad(x, p, st, st[:5], x, x)
    with pytest.raises(evox.EvoxError):
        evox.evox_xent(x, st, torch.zeros(2))
    with pytest.raises(evox.EvoxError):
        evox.evox_xent(x, st.int(), torch.zeros(2, dtype=torch.float64))
