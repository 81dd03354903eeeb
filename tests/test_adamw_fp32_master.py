"""fp32 parameters are their own master: the library refuses another, as the binding does."""
import ctypes

import pytest

from test_mix_abi import P, adam, evox, plan, step, tensor  # noqa: F401


@pytest.mark.parametrize("bits", [32, 8])
def test_plan_refuses_a_master_of_fp32(evox, bits):  # noqa: F811
    for ts in ([tensor(evox, master=P)], [tensor(evox, master=P), tensor(evox, p=2 * P, master=2 * P)], [tensor(evox, master=P, rows=0)]):
        assert plan(evox, *ts, dtype=evox.F32, bits=bits) == evox.EINVAL
        assert b"own master" in evox.lib().evox_last_error()
    # in 16 bits it is looked at further
    assert plan(evox, tensor(evox, master=P), dtype=evox.BF16, bits=bits, table=None) == evox.EINVAL
    assert b"scratch" in evox.lib().evox_last_error()


@pytest.mark.parametrize("bits", [32, 8])
def test_step_refuses_a_plan_of_fp32_with_a_master(evox, bits):  # noqa: F811
    p = evox.AdamPlan(table=P, count=1, tiles=1, dtype=evox.F32, bits=bits, master=1)
    assert evox.lib().evox_adamw(ctypes.byref(adam(evox)), ctypes.byref(p), None, None) == evox.EINVAL
    assert b"plan" in evox.lib().evox_last_error()  # (not for the clock that is missing too)
