"""The traffic figures that bench.py reports carry the library version that they were measured on: the file of the runs says the same."""
import ast
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def traffic():
    tree = ast.parse(open(os.path.join(ROOT, "bench.py")).read())
    return next(ast.literal_eval(node.value) for node in tree.body
                if isinstance(node, ast.Assign) and [getattr(t, "id", None) for t in node.targets] == ["TRAFFIC"])


@pytest.mark.parametrize("which", ["prefill", "decode"])
def test_the_stamp_is_the_version_of_the_runs(which):
    t = traffic()[which]
    runs = open(os.path.join(ROOT, t["source"])).read()
    said = re.search(r"`bench\.py` reports the first line as.*?stamped with library version (\d+)", runs, re.S)
    assert int(said.group(1)) == t["library_version"]
    first = re.search(r"library version (\d+)", runs)      # the heading's
    assert int(first.group(1)) == t["library_version"]
    assert t["kernel"] in runs.replace("`", "")
