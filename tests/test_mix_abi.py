"""Host-side refusals of the mixtures' operators and of the optimizer's step (validation
runs before any HIP call, so no GPU is needed)."""
import ctypes
import math
import os

import pytest


@pytest.fixture(scope="module")
def evox():
    import paper_2301_12457_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2301_12457_amd import build
        build.build()
    return m


P = 0x1000  # never dereferenced
BIG = 1 << 40


def call(evox, name, struct, *args):
    return getattr(evox.lib(), name)(ctypes.byref(struct) if struct is not None else None, *args, None)


def test_struct_layouts(evox):
    assert ctypes.sizeof(evox.Choice) == 8 + 5 * 8 and evox.Choice.T.offset == 8
    assert ctypes.sizeof(evox.Slots) == 8 + 9 * 8 and evox.Slots.ldds.offset == 72
    assert ctypes.sizeof(evox.Parameter) == 12 * 8 and evox.Parameter.rows.offset == 56
    assert ctypes.sizeof(evox.Adam) == 5 * 8 + 8 and evox.Adam.lr_dev.offset == 40
    assert ctypes.sizeof(evox.AdamPlan) == 3 * 8 + 16 and evox.AdamPlan.dtype.offset == 24


def choice(evox, **kw):
    return evox.Choice(**dict(dict(dtype=evox.F32, over=evox.GATE_ALL, T=6, G=5, k=2, ldz=5, lddz=5), **kw))


BAD_CHOICE = [dict(dtype=3), dict(dtype=-1), dict(over=2), dict(over=-1), dict(G=0), dict(G=32_769, ldz=BIG), dict(k=0),
              dict(k=6), dict(k=33, G=40, ldz=40), dict(T=-1), dict(T=1 << 30), dict(T=1 << 62), dict(ldz=4), dict(ldz=1 << 31)]


def gate(evox, c, z=P, ids=P, w=P):
    return call(evox, "evox_gate", c, z, ids, w)


def gate_grad(evox, c, z=P, ids=P, w=P, dw=P, dz=P):
    return call(evox, "evox_gate_grad", c, z, ids, w, dw, dz)


@pytest.mark.parametrize("kw", BAD_CHOICE)
def test_gate_refuses(evox, kw):
    assert gate(evox, choice(evox, **kw)) == evox.EINVAL
    assert gate_grad(evox, choice(evox, **kw)) == evox.EINVAL
    assert len(evox.lib().evox_last_error()) > 5


def test_gate_refuses_operands(evox):
    c = choice(evox)
    assert gate(evox, None) == evox.EINVAL and gate_grad(evox, None) == evox.EINVAL
    for k in ("z", "ids", "w"):
        assert gate(evox, c, **{k: None}) == evox.EINVAL
        assert gate(evox, c, **{k: P + 2}) == evox.EALIGN
    assert gate(evox, choice(evox, dtype=evox.F16), z=P + 1) == evox.EALIGN
    for k in ("z", "ids", "w", "dw", "dz"):
        assert gate_grad(evox, c, **{k: None}) == evox.EINVAL
        assert gate_grad(evox, c, **{k: P + 2}) == evox.EALIGN
    assert gate_grad(evox, choice(evox, lddz=4)) == evox.EINVAL
    empty = choice(evox, T=0)
    assert gate(evox, empty, None, None, None) == evox.OK and gate_grad(evox, empty, None, None, None, None, None) == evox.OK


def slots(evox, **kw):
    return evox.Slots(**dict(dict(dtype=evox.F32, T=6, k=2, G=3, M=12, D=5, ldx=5, ldy=5, lds=5, ldds=5), **kw))


def route(evox, p, ids=P, off=P, pos=P, src=P, scratch=P, nbytes=BIG):
    return call(evox, "evox_route", p, ids, off, pos, src, scratch, nbytes)


def dispatch(evox, p, x=P, pos=P, w=P, xs=P):
    return call(evox, "evox_dispatch", p, x, pos, w, xs)


def combine(evox, p, xs=P, pos=P, w=P, r=P, y=P):
    return call(evox, "evox_combine", p, xs, pos, w, r, y)


def combine_grad(evox, p, xs=P, pos=P, w=P, dy=P, dxs=P, dw=P):
    return call(evox, "evox_combine_grad", p, xs, pos, w, dy, dxs, dw)


def test_route_refuses(evox):
    need = evox.lib().evox_route_scratch_bytes(ctypes.byref(slots(evox)))
    assert need > 0
    for kw in (dict(k=0), dict(k=1025), dict(T=-1), dict(T=1 << 30), dict(G=0), dict(G=(1 << 20) + 1)):
        assert route(evox, slots(evox, **kw)) == evox.EINVAL, kw
        assert evox.lib().evox_route_scratch_bytes(ctypes.byref(slots(evox, **kw))) == 0
    assert route(evox, None) == evox.EINVAL and evox.lib().evox_route_scratch_bytes(None) == 0
    for k in ("ids", "off", "pos", "scratch"):
        assert route(evox, slots(evox), **{k: None}) == evox.EINVAL
    for k in ("ids", "off", "pos", "src"):
        assert route(evox, slots(evox), **{k: P + 2}) == evox.EALIGN
    assert route(evox, slots(evox), scratch=P + 16) == evox.EALIGN
    assert route(evox, slots(evox), nbytes=need - 1) == evox.ENOSPC


def test_slots_refuse(evox):
    for f in (dispatch, combine, combine_grad):
        assert f(evox, None) == evox.EINVAL
        for kw in (dict(dtype=5), dict(k=0), dict(k=1025), dict(T=-1), dict(T=1 << 30), dict(M=-1), dict(M=1 << 31), dict(D=0),
                   dict(D=(1 << 20) + 1), dict(lds=4), dict(ldx=4), dict(ldx=1 << 31)):
            assert f(evox, slots(evox, **kw)) == evox.EINVAL, kw
    assert combine(evox, slots(evox, ldy=4)) == evox.EINVAL and combine_grad(evox, slots(evox, ldds=4)) == evox.EINVAL
    for f, need, all_ in ((dispatch, "x pos xs", "x pos w xs"), (combine, "xs pos y", "xs pos w r y"),
                          (combine_grad, "xs pos dy", "xs pos w dy dxs dw")):
        for k in need.split():
            assert f(evox, slots(evox), **{k: None}) == evox.EINVAL, k
        for k in all_.split():
            assert f(evox, slots(evox), **{k: P + 2}) == evox.EALIGN, k
    bf = slots(evox, dtype=evox.BF16)
    assert dispatch(evox, bf, x=P + 1) == evox.EALIGN and combine(evox, bf, w=P + 2) == evox.EALIGN
    none = slots(evox, T=0)
    assert dispatch(evox, none, None, None, None, None) == evox.OK
    assert combine(evox, none, None, None, None, None, None) == evox.OK
    assert combine_grad(evox, slots(evox), None, None, None, None, None, None) == evox.OK  # nothing asked for


def tensor(evox, **kw):
    return evox.Parameter(**dict(dict(p=P, g=P, m=P, v=P, m_scale=P, v_scale=P, master=None, rows=3, n=5, ldp=5, ldg=5, lds=5), **kw))


def plan(evox, *ts, dtype=0, bits=32, count=None, table=P, nbytes=BIG, out=True):
    p = evox.AdamPlan()
    return evox.lib().evox_adamw_plan(dtype, bits, (evox.Parameter * len(ts))(*ts) if ts else None, len(ts) if count is None else count,
                                      table, nbytes, ctypes.byref(p) if out else None, None)


def test_plan_refuses(evox):
    need = evox.lib().evox_adamw_table_bytes
    assert need(1) > 0 and need(0) > 0 and need(-1) == 0 and need((1 << 20) + 1) == 0
    ok = tensor(evox)
    for kw in (dict(dtype=3), dict(bits=16), dict(count=-1), dict(count=(1 << 20) + 1), dict(out=False), dict(table=None)):
        assert plan(evox, ok, **kw) == evox.EINVAL, kw
    assert plan(evox, count=1) == evox.EINVAL
    assert plan(evox, ok, table=P + 16) == evox.EALIGN and plan(evox, ok, nbytes=need(1) - 1) == evox.ENOSPC
    for kw in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(rows=-1), dict(rows=1 << 31), dict(n=-1), dict(n=1 << 39),
               dict(ldp=4), dict(ldg=4), dict(lds=4), dict(ldp=1 << 60), dict(rows=1 << 30, n=1 << 20, ldp=1 << 20, ldg=1 << 20, lds=1 << 20)):
        assert plan(evox, tensor(evox, **kw)) == evox.EINVAL, kw
    for k in ("p", "g", "m", "v", "master"):
        assert plan(evox, tensor(evox, **{k: P + 2})) == evox.EALIGN
    for k in ("m_scale", "v_scale"):
        assert plan(evox, tensor(evox, **{k: None}), bits=8) == evox.EINVAL
        assert plan(evox, tensor(evox, **{k: P + 1}), bits=8) == evox.EALIGN
    # a master for all or for none; no tensor twice; not too many elements in all
    assert plan(evox, tensor(evox, master=P), tensor(evox, p=2 * P)) == evox.EINVAL
    assert plan(evox, *[tensor(evox, p=P * (i % 40 + 1)) for i in range(41)]) == evox.EINVAL
    assert b"twice" in evox.lib().evox_last_error()
    big = dict(rows=1, n=1 << 38)
    assert plan(evox, *[tensor(evox, p=P * (i + 1), **big) for i in range(40)]) == evox.EINVAL
    assert b"together" in evox.lib().evox_last_error()


def adam(evox, **kw):
    return evox.Adam(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1), **kw))


def step(evox, a, clock=P, **kw):
    p = evox.AdamPlan(**dict(dict(table=P, count=1, tiles=1, dtype=0, bits=32, master=0), **kw))
    return evox.lib().evox_adamw(ctypes.byref(a) if a else None, ctypes.byref(p), clock, None)


@pytest.mark.parametrize("kw", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0),
                                dict(eps=1e-60), dict(eps=math.inf), dict(eps=math.nan), dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e300),
                                dict(weight_decay=math.nan)])
def test_step_refuses(evox, kw):
    assert step(evox, adam(evox, **kw)) == evox.EINVAL


def test_step_refuses_plans(evox):
    a = adam(evox)
    assert step(evox, None) == evox.EINVAL and evox.lib().evox_adamw(ctypes.byref(a), None, P, None) == evox.EINVAL
    for kw in (dict(table=None), dict(count=-1), dict(tiles=-1), dict(tiles=1 << 31), dict(dtype=3), dict(bits=0)):
        assert step(evox, a, **kw) == evox.EINVAL, kw
    assert step(evox, a, clock=None) == evox.EINVAL and step(evox, a, clock=P + 4) == evox.EALIGN
    assert step(evox, adam(evox, lr_dev=P + 2)) == evox.EALIGN
