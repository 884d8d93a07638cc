"""The block example gives every library call the caller's current stream."""
import ast
import inspect

import paper_2409_03864_b200 as tdx
from paper_2409_03864_b200 import run_decay_block


def test_no_library_call_is_left_on_the_default_stream():
    def takes_stream(name):
        f = getattr(tdx, name, None)
        return inspect.isfunction(f) and "stream" in inspect.signature(f).parameters

    direct = [n for n in ast.walk(ast.parse(inspect.getsource(run_decay_block))) if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute)
              and isinstance(n.func.value, ast.Name) and n.func.value.id == "tdx" and takes_stream(n.func.attr)]
    assert [n.func.attr for n in direct if not any(k.arg == "stream" for k in n.keywords)] == []
