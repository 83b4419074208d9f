"""Modules that can be run as scripts bind every name before their script part: it is the last statement of the file."""
import ast
import glob
import os

import pytest

from paper_2401_06706_b200 import build

FILES = sorted(os.path.relpath(f, build.ROOT) for pattern in ("*.py", "paper_2401_06706_b200/*.py", "oracle/*.py", "perf/*.py")
               for f in glob.glob(os.path.join(build.ROOT, pattern)))


def _is_script_part(node):
    return isinstance(node, ast.If) and "__name__" in {n.id for n in ast.walk(node.test) if isinstance(n, ast.Name)}


@pytest.mark.parametrize("name", FILES)
def test_nothing_follows_the_script_part(name):
    with open(os.path.join(build.ROOT, name)) as f:
        body = ast.parse(f.read()).body
    at = [i for i, node in enumerate(body) if _is_script_part(node)]
    assert at in ([], [len(body) - 1])
