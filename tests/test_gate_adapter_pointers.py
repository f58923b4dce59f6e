"""Pointers that are no multiple of their type's size are refused before a device is touched: a kernel could not read through them."""
from ctypes import byref, c_size_t

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2608_15383_b200 import binding, build
    build.build()
    binding.lib()
    return binding


P, MB = 1 << 30, 1 << 20                                                   # aligned addresses that are never used


@pytest.mark.parametrize("name", ["bias", "addend", "balance", "ids", "weights"])
def test_gate_on_hidden_states(B, name):
    at = dict(bias=P, addend=P + MB, balance=P + 2 * MB, ids=P + 3 * MB, weights=P + 4 * MB)
    for off in (1, 2, 3):
        p = {**at, name: at[name] + off}
        rc = B.lib().exmoe_route_gated(byref(B.exmoe_shape(64, 128, 8, 2, 128)), byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0)), P + 5 * MB, P + 6 * MB, p["bias"], p["addend"],
                                       p["balance"], 1, p["ids"], p["weights"], None)
        assert rc == B.EXMOE_ERR_ARG, off


@pytest.mark.parametrize("name", ["logits", "balance", "ids", "weights"])
@pytest.mark.parametrize("type", [0, 1])
def test_gate_on_logits(B, name, type):
    at = dict(logits=P, balance=P + MB, ids=P + 2 * MB, weights=P + 3 * MB)
    for off in (1, 3) if name == "logits" and type else (1, 2, 3):
        p = {**at, name: at[name] + off}
        rc = B.lib().exmoe_gate_logits(byref(B.exmoe_shape(0, 0, 8, 2, 0)), byref(B.exmoe_gate(0, 1, 1, 0, 0, 1.0)), p["logits"], type, 8, p["balance"], 2, p["ids"],
                                       p["weights"], None)
        assert rc == B.EXMOE_ERR_ARG, off


@pytest.mark.parametrize("name", ["scale", "base", "out"])
@pytest.mark.parametrize("type", [0, 1])
def test_adapters(B, name, type):
    at = dict(scale=P, base=P + MB, out=P + 2 * MB)
    for off in (1, 3) if name != "scale" and type else (1, 2, 3):
        p = {**at, name: at[name] + off}
        rc = B.lib().exmoe_lora(byref(B.exmoe_lora_shape(4, 64, 32, 8)), P + 3 * MB, P + 4 * MB, 64, P + 5 * MB, P + 6 * MB, p["scale"], 16, p["base"], 32, p["out"], 32, type, None)
        assert rc == B.EXMOE_ERR_ARG, off


def test_adapter_ids_and_their_bytes(B):
    for off in (1, 2, 3):
        assert B.lib().exmoe_lora_plan(P + off, 5, 4, P + MB, None) == B.EXMOE_ERR_ARG
    n = c_size_t()
    assert B.lib().exmoe_lora_plan_bytes(5, 4, byref(n)) == B.EXMOE_OK and n.value
