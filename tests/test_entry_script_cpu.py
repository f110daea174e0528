"""__graft_entry__.py run as a script has all of the module's functions when it calls smoke()."""
import ast
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_everything_is_defined_before_the_script_part():
    with open(os.path.join(ROOT, "__graft_entry__.py")) as f:
        body = ast.parse(f.read()).body
    script = [i for i, node in enumerate(body) if isinstance(node, ast.If) and "__main__" in ast.dump(node.test)]
    assert len(script) == 1
    late = [node.name for node in body[script[0] + 1:] if isinstance(node, (ast.FunctionDef, ast.ClassDef))]
    assert not late, "defined after the script part has run: %s" % late
