"""The build and smoke entry points need no test runner: every module of the tests that they import loads without pytest."""
import ast
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_entry_points_load_without_pytest():
    with open(os.path.join(ROOT, "__graft_entry__.py")) as f:
        tree = ast.parse(f.read())
    imports = [n for n in ast.walk(tree) if isinstance(n, ast.ImportFrom) and n.module.startswith(("tests", "oracle"))]
    assert imports
    code = "import sys; sys.modules['pytest'] = None\n" + "\n".join(ast.unparse(n) for n in imports)
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-1000:]
