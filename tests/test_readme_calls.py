"""The Python of README.md against the signatures it calls: names exist, arguments
bind, and a variable that is named for a role is passed in that role."""
import ast
import inspect
import os
import re

import pytest

from tests.conftest import ROOT

zf = pytest.importorskip("paper_2505_12242_amd")


def blocks():
    """The indented Python blocks that use the package."""
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    out = re.findall(r"(?:^    .*\n|^\n)+", text, re.M)
    return [inspect.cleandoc("\n" + b) for b in out if "zf." in b and "python " not in b]


def calls():
    for b in blocks():
        for node in ast.walk(ast.parse(b)):
            if isinstance(node, ast.Call):
                name = ast.unparse(node.func)
                if name.startswith("zf."):
                    yield name, node


def resolve(name):
    obj = zf
    for part in name.split(".")[1:]:
        obj = getattr(obj, part)
    return obj


def test_calls_bind():
    found = list(calls())
    assert {"zf.rmsnorm", "zf.matmul_fp8", "zf.AdamWBuffers.fresh"} <= {n for n, _ in found}
    for name, node in found:
        bound = inspect.signature(resolve(name)).bind(
            *node.args, **{k.arg: k.value for k in node.keywords})
        for role, value in bound.arguments.items():
            if not isinstance(value, ast.Name):
                continue
            words = set(value.id.split("_"))
            if "grad" in words:  # gain_grad: a gradient, not the parameter itself
                assert role in ("grad", "grads", "grad_slots"), (name, role, value.id)
            if role == "grad":
                assert "grad" in words, (name, role, value.id)
