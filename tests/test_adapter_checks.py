"""The binding's checks of arguments stay where python -O takes assert statements out (no GPU)."""
import ast
import os
import subprocess
import sys

import paper_2206_10620_amd as pp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import types
import torch
import paper_2206_10620_amd as pp
from paper_2206_10620_amd import pp_adapter as binding

host = torch.zeros((4, 8), dtype=torch.float16)
held = torch.zeros(pp.pp_act8_bytes(4, 8), dtype=torch.uint8)
# a bank as its methods see it, without one on a device
bank = types.SimpleNamespace(handle=None, m=4, k=4, slots=1, max_rank=4, dtype=pp.PP_F16, device=torch.device("cuda", 0), _state_bytes=lambda n: (16, 16))
for name in ("_slots_of", "load"):
    setattr(bank, name, types.MethodType(getattr(pp.AdapterBank, name), bank))
calls = {
    "pack": lambda: pp.act8_pack(host),
    "buffer size": lambda: pp.Act8(held[1:], 4, 8, pp.PP_F16),
    "buffer device": lambda: pp.Act8(held, 4, 8, pp.PP_F16),
    "lengths": lambda: pp.pp_adapter_load_many(None, [0, 1], [1], [1.0], [16], [16]),
    "load": lambda: pp.AdapterBank.load(bank, 0, host, host, 1.0),
    "load_many, one": lambda: pp.AdapterBank.load_many(bank, [0], [host], [host], [1.0]),
    "load_many, two": lambda: pp.AdapterBank.load_many(bank, [0, 0], [host, host], [host, host], [1.0, 1.0]),
    "load_many lengths": lambda: pp.AdapterBank.load_many(bank, [0, 0], [host], [host], [1.0]),
    "project": lambda: pp.AdapterBank.project(bank, host, host),
    "run": lambda: pp.AdapterBank.run(bank, None, host, host),
    "grad_input": lambda: pp.AdapterBank.grad_input(bank, None, host, host),
    "grad_weights": lambda: pp.AdapterBank.grad_weights(bank, host, held, host, held, host, host),
    "slots": lambda: bank._slots_of(host, 8),
}
for name, call in calls.items():
    try:
        call()
    except AssertionError:
        print("refused", name)
    else:
        print("ACCEPTED", name)
"""


def test_arguments_are_checked_without_assert_statements_too():
    for flags in ([], ["-O"]):
        r = subprocess.run([sys.executable, *flags, "-c", CALLS], capture_output=True, text=True, cwd=ROOT, timeout=300)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == 13 and all(line.startswith("refused ") for line in lines), (flags, r.stdout[-2000:], r.stderr[-2000:])


def test_the_binding_has_no_assert_statement():
    path = os.path.join(ROOT, "paper_2206_10620_amd", "pp_adapter.py")
    assert not [node.lineno for node in ast.walk(ast.parse(open(path).read())) if isinstance(node, ast.Assert)]
    assert pp.AdapterBank.__module__.endswith("pp_adapter")
