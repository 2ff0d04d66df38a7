"""The binding's classes, read as source (no GPU, no library)."""
import ast
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = [os.path.join("paper_2408_05646_b200", f) for f in ("binding.py", "build.py", "synth.py")] + ["bench.py", "__graft_entry__.py"]


def test_no_class_or_module_defines_a_name_twice():
    """Python keeps the last definition and says nothing: an earlier one is out of reach, whatever it does."""
    for path in SOURCES:
        tree = ast.parse(open(os.path.join(ROOT, path)).read())
        for scope in [tree] + [n for n in ast.walk(tree) if isinstance(n, ast.ClassDef)]:
            names = [n.name for n in scope.body if isinstance(n, (ast.FunctionDef, ast.ClassDef))]
            twice = sorted({n for n in names if names.count(n) > 1})
            assert not twice, f"{path}, {getattr(scope, 'name', 'module')}: {twice}"
