"""The state-space layer example gives every library call the caller's current stream."""
import ast
import inspect

import pytest
import torch

import paper_2409_03864_b200 as tdx
from paper_2409_03864_b200 import run_ssm_layer


def takes_stream(name):
    f = getattr(tdx, name, None)
    return inspect.isfunction(f) and "stream" in inspect.signature(f).parameters


def test_no_library_call_is_left_on_the_default_stream():
    direct = [n for n in ast.walk(ast.parse(inspect.getsource(run_ssm_layer))) if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute)
              and isinstance(n.func.value, ast.Name) and n.func.value.id == "tdx" and takes_stream(n.func.attr)]
    assert [n.func.attr for n in direct if not any(k.arg == "stream" for k in n.keywords)] == []


def test_calls_get_the_current_stream_and_errors_are_raised(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "the caller's")
    seen = []
    run_ssm_layer._call(lambda *a, stream=None: seen.append((a, stream)) or 0, 1, 2)
    assert seen == [((1, 2), "the caller's")]
    with pytest.raises(tdx.TdxError):
        run_ssm_layer._call(lambda stream=None: tdx.TDX_ERR_INVALID_ARG)
