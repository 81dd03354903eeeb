"""The binding of the mixtures' operators and of the optimizer, on the host: tensors that
say they are on the GPU and a library that notes its calls stand in for both."""
import types

import pytest
import torch

from host_tensors import Library, Streams, gpu, on_host_device


@pytest.fixture
def evox(monkeypatch):
    import paper_2301_12457_amd as m
    L = Library()
    monkeypatch.setattr(m, "lib", lambda: L)
    m.calls = L.calls
    on_host_device(m, monkeypatch)
    return m


def new(*shape, **kw):
    return gpu(torch.zeros(*shape, **kw))


I32 = dict(dtype=torch.int32)


def arguments():
    ids, pos, w = new(6, 2, **I32), new(6, 2, **I32), new(6, 2)
    return {"evox_gate": dict(logits=new(6, 5), ids=ids, w=w),
            "evox_gate_grad": dict(logits=new(6, 5), ids=ids, w=w, dw=new(6, 2), dz=new(6, 5)),
            "evox_route": dict(ids=ids, off=new(6, **I32), pos=pos, src=new(12, **I32), scratch=new(4096)),
            "evox_dispatch": dict(x=new(6, 7), pos=pos, xs=new(12, 7), w=w),
            "evox_combine": dict(xs=new(12, 7), pos=pos, y=new(6, 7), w=w, r=new(6, 7)),
            "evox_combine_grad": dict(xs=new(12, 7), pos=pos, dy=new(6, 7), w=w, dxs=new(12, 7), dw=new(6, 2))}


OPTIONAL = {"src", "scratch", "w", "r", "dxs", "dw", "xs"}


@pytest.mark.parametrize("name", sorted(arguments()))
def test_calls_reach_the_library(evox, name):
    getattr(evox, name)(**arguments()[name])
    assert evox.calls[-1][0] == name and evox.calls[-1][1][-1] == 7
    getattr(evox, name)(**arguments()[name], stream=types.SimpleNamespace(cuda_stream=9))
    assert evox.calls[-1][1][-1] == 9


def test_what_the_structures_say(evox):
    a = arguments()
    wide = lambda rows, n: new(rows, n + 4)[:, :n]
    evox.evox_gate(wide(6, 5), a["evox_gate"]["ids"], a["evox_gate"]["w"], over=evox.GATE_ALL)
    p = evox.calls[-1][1][0]._obj
    assert (p.dtype, p.over, p.T, p.G, p.k, p.ldz) == (evox.F32, 1, 6, 5, 2, 9)
    evox.evox_route(**a["evox_route"])
    p = evox.calls[-1][1][0]._obj
    assert (p.T, p.k, p.G) == (6, 2, 5)
    evox.evox_combine_grad(wide(11, 7), a["evox_combine"]["pos"], wide(6, 7), dxs=new(11, 9)[:, :7])
    p = evox.calls[-1][1][0]._obj
    assert (p.T, p.k, p.M, p.D, p.ldx, p.lds, p.ldds) == (6, 2, 11, 7, 11, 11, 9)
    evox.evox_combine(wide(11, 7), a["evox_combine"]["pos"], wide(6, 7), r=new(6, 7))
    p = evox.calls[-1][1][0]._obj
    assert (p.M, p.ldx, p.ldy, p.lds) == (11, 7, 11, 11)


def odd(*shape, **kw):
    """Of this shape, its last dimension not dense."""
    return new(*shape[:-1], 2 * shape[-1], **kw)[..., ::2]


GATE = [("logits", new(6), r"must be \[T, G\]"), ("logits", odd(6, 5), "logits: rows are not dense"), ("logits", new(6, 5).double(), "float64"),
        ("logits", torch.zeros(6, 5), "GPU's memory"), ("ids", new(6, **I32), r"must be \[T, G\]"), ("ids", new(6, 2), "ids: a dense int32"),
        ("ids", new(5, 2, **I32), "ids: a dense int32"), ("ids", odd(6, 2, **I32), "ids: a dense int32"),
        ("ids", new(6, 2, dtype=torch.int64), "ids: a dense int32"), ("w", new(6, 3), "w: a dense float32"),
        ("w", new(6, 2).half(), "w: a dense float32"), ("w", gpu(torch.zeros(6, 2), 1), "w: a dense float32")]
GRAD = [("dw", new(5, 2), "dw: a dense float32"), ("dw", new(6, 2).double(), "dw: a dense float32"), ("dz", new(6, 4), "dz has shape"),
        ("dz", odd(6, 5), "dz: rows are not dense"), ("dz", new(6, 5).half(), "dz: torch.float16")]
ROUTE = [("ids", new(12, **I32), r"must be \[T, k\]"), ("ids", new(6, 2), "ids: a dense int32"), ("ids", torch.zeros(6, 2, **I32), "GPU's memory"),
         ("off", new(1, **I32), r"off \[G \+ 1\]"), ("off", new(6), "off: a dense int32"), ("off", gpu(torch.zeros(6, **I32), 1), "off: a dense int32"),
         ("pos", new(12, **I32), "pos: a dense int32"), ("pos", new(6, 3, **I32), "pos: a dense int32"), ("src", new(11, **I32), "src: a dense int32"),
         ("src", new(6, 2, **I32), "src: a dense int32"), ("scratch", odd(4096), "scratch: a dense")]
DISPATCH = [("x", new(6), r"must be \[T, D\]"), ("x", odd(6, 7), "x: rows are not dense"), ("x", new(5, 7), "pos: a dense int32"),
            ("pos", new(12, **I32), r"must be \[T, D\]"), ("pos", new(6, 2), "pos: a dense int32"), ("xs", new(12, 6), "xs has shape"),
            ("xs", new(12, 7).half(), "xs: torch.float16"), ("xs", odd(12, 7), "xs: rows are not dense"), ("xs", new(84), r"must be \[T, D\]"),
            ("w", new(6, 3), "w: a dense float32"), ("w", new(6, 2).bfloat16(), "w: a dense float32")]
COMBINE = [("y", odd(6, 7), "y: rows are not dense"), ("y", new(6, 7).half(), "xs: torch.float32"), ("r", new(6, 6), "r has shape"),
           ("r", new(6, 7).half(), "r: torch.float16"), ("xs", new(12, 8), "xs has shape"), ("pos", new(5, 2, **I32), "pos: a dense int32")]
CGRAD = [("dy", odd(6, 7), "dy: rows are not dense"), ("dxs", new(11, 7), "dxs has shape"), ("dxs", new(84), r"dxs must be \[M, D\]"),
         ("dxs", new(12, 7).half(), "dxs: torch.float16"), ("dw", new(6, 3), "dw: a dense float32"), ("xs", None, "xs is required")]
CASES = [(n, *c) for n, cases in (("evox_gate", GATE), ("evox_gate_grad", GATE[:6] + GRAD), ("evox_route", ROUTE), ("evox_dispatch", DISPATCH),
                                  ("evox_combine", COMBINE), ("evox_combine_grad", CGRAD)) for c in cases]


@pytest.mark.parametrize("name,what,value,words", CASES)
def test_refusals_and_their_reasons(evox, name, what, value, words):
    with pytest.raises(evox.EvoxError, match=words) as e:
        getattr(evox, name)(**dict(arguments()[name], **{what: value}))
    assert e.value.code == evox.EINVAL and not any(n == name for n, _ in evox.calls)


@pytest.mark.parametrize("name,what", [(n, w) for n, a in arguments().items() for w in a if w not in OPTIONAL or n == "evox_gate"
                                       or n == "evox_gate_grad" or (n, w) in (("evox_dispatch", "xs"), ("evox_combine", "xs"))])
def test_none_for_what_is_needed(evox, name, what):
    with pytest.raises(evox.EvoxError, match=f"{what} is required"):
        getattr(evox, name)(**dict(arguments()[name], **{what: None}))


@pytest.mark.parametrize("name", sorted(arguments()))
def test_another_device(evox, monkeypatch, name):
    on_host_device(evox, monkeypatch, 1)
    with pytest.raises(evox.EvoxError, match="the current device is 1"):
        getattr(evox, name)(**arguments()[name])
    on_host_device(evox, monkeypatch, 0)
    with pytest.raises(evox.EvoxError, match="the stream's 1"):
        getattr(evox, name)(**arguments()[name], stream=types.SimpleNamespace(cuda_stream=5, device=torch.device("cuda", 1)))
    assert all(n.endswith("_bytes") for n, _ in evox.calls)


def test_scratch_of_the_call_s_stream(evox, monkeypatch):
    streams = Streams(monkeypatch)
    a = arguments()["evox_route"]
    evox.evox_route(a["ids"], a["off"], a["pos"], stream=streams.stream(2))
    assert [s.cuda_stream for s in streams.allocated] == [2] and evox.calls[-1][1][-1] == 2


@pytest.fixture
def here(evox, monkeypatch):
    """States that are made on the host count as the GPU's."""
    real = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: gpu(real(*a, **k)))
    return evox


def planned(evox):
    """The tensors of the last plan."""
    name, args = [c for c in evox.calls if c[0] == "evox_adamw_plan"][-1]
    assert args[5] == 4096 and args[7] == 7
    return args[0], args[1], list(args[2])


def test_optimizer_s_tensors(here):
    evox = here
    X, D = new(5, 700), new(5, 710)
    params = [new(3, 4), X[:, 1:4], X[:, 10:610].unflatten(1, (2, 300)), new(9)]
    grads = [new(3, 4), D[:, 1:4], D[:, 10:610].unflatten(1, (2, 300)), new(9)]
    opt = evox.AdamW(params, grads, lr=0.5, betas=(0.8, 0.7), eps=0.1, weight_decay=0.3, bits=8)
    s = opt.state
    assert sorted(s) == ["m", "m_scale", "t", "v", "v_scale"] and s["m"].dtype == torch.float8_e4m3fn
    assert s["m"].numel() == 12 + 15 + 3000 + 9 and s["v_scale"].numel() == 1 + 5 + 5 * 3 + 1
    dtype, bits, t = planned(evox)
    assert (dtype, bits) == (evox.F32, 8)
    assert [(x.rows, x.n, x.ldp, x.ldg, x.lds) for x in t] == [(1, 12, 12, 12, 12), (5, 3, 700, 710, 3), (5, 600, 700, 710, 600), (1, 9, 9, 9, 9)]
    assert [x.m - t[0].m for x in t] == [0, 12, 27, 3027] and [x.v_scale - t[0].v_scale for x in t] == [0, 4, 24, 84]
    assert t[1].p == params[1].data_ptr() and t[1].g == grads[1].data_ptr() and t[0].master is None
    opt.step()
    name, args = evox.calls[-1]
    a = args[0]._obj
    assert name == "evox_adamw" and args[1]._obj is opt._plan and args[2] == s["t"].data_ptr() and args[3] == 7
    assert (a.lr, a.beta1, a.beta2, a.eps, a.weight_decay, a.lr_dev) == (0.5, 0.8, 0.7, 0.1, 0.3, None)
    opt.lr = lr = new(1)
    opt.step(stream=types.SimpleNamespace(cuda_stream=3))
    assert evox.calls[-1][1][-1] == 3 and evox.calls[-1][1][0]._obj.lr_dev == lr.data_ptr()
    opt.lr = 0.25
    opt.step()
    assert evox.calls[-1][1][0]._obj.lr_dev is None and evox.calls[-1][1][0]._obj.lr == 0.25


def test_optimizer_s_master(here):
    p = new(2, 5).bfloat16() + 1
    opt = here.AdamW([p, gpu(p.clone())], [new(2, 5).bfloat16()] * 2, master=True)
    assert opt.state["master"].tolist() == [1.0] * 20 and opt.state["m"].dtype == torch.float32
    t = planned(here)[2]
    assert [x.master - t[0].master for x in t] == [0, 40]
    # of parameters that a program trains, no part of their graph
    leaf = p.clone().requires_grad_()
    opt = here.AdamW([gpu(leaf)], [new(2, 5).bfloat16()], master=True)
    assert not opt.state["master"].requires_grad


def test_scalar_gradient_rows(evox):
    a = arguments()["evox_combine_grad"]
    with pytest.raises(evox.EvoxError, match=r"dxs must be \[M, D\]"):
        evox.evox_combine_grad(**dict(a, dxs=gpu(torch.tensor(1.0))))


@pytest.mark.parametrize("params,grads,kw,words", [
    ([], [], {}, "0 parameters"), ([new(3)], [], {}, "1 parameters and 0"), ([new(3)], [new(4)], {}, r"params\[0\] has shape"),
    ([new(3), new(3).half()], [new(3), new(3).half()], {}, r"params\[1\]: torch.float16"), ([new(3)], [new(3).half()], {}, r"grads\[0\]"),
    ([new(3)], [gpu(torch.zeros(3), 1)], {}, r"grads\[0\]"), ([odd(3, 4)], [new(3, 4)], {}, r"params\[0\]: rows are not dense"),
    ([new(3, 4)], [odd(3, 4)], {}, r"grads\[0\]: rows are not dense"), ([odd(4)], [new(4)], {}, r"params\[0\]: rows"),
    ([new(3, 4, 5).transpose(1, 2)], [new(3, 5, 4)], {}, "rows are not dense"), ([torch.zeros(3)], [torch.zeros(3)], {}, "GPU's memory"),
    ([new(3)], [new(3)], dict(bits=16), "bits = 16"), ([new(3)], [new(3)], dict(master=True), "own master"), ([new(3).double()], [new(3).double()], {}, "float64"),
    ([gpu(torch.tensor(1.0))], [gpu(torch.tensor(1.0))], {}, "has shape")])
def test_optimizer_refuses(here, params, grads, kw, words):
    with pytest.raises(here.EvoxError, match=words):
        here.AdamW(params, grads, **kw)
    assert not any(n == "evox_adamw_plan" for n, _ in here.calls)


def test_optimizer_refuses_rates_and_devices(here, monkeypatch):
    opt = here.AdamW([new(3)], [new(3)], lr=new(2))
    with pytest.raises(here.EvoxError, match="lr: a dense float32 tensor of 1"):
        opt.step()
    opt.lr = 1.0
    on_host_device(here, monkeypatch, 1)
    with pytest.raises(here.EvoxError, match="the current device is 1"):
        opt.step()
    assert not any(n == "evox_adamw" for n, _ in here.calls)
